// Beam search: the best continuations of every prompt's beams, and caches that follow their beams.
#include "thk_step.h"

#include <math.h>

#include <algorithm>

namespace thk {
namespace {

typedef unsigned long long u64;

// ---- selection ----------------------------------------------------------------------------
// A row of logits is cut into pieces, a block each, whose waves go over a part of theirs once: a running sum of exp(x - r) per lane, r what the
// lane's largest element was or not much less, and each lane's largest element of every tile, which waits in LDS.  Then the K-th of the block's lanes'
// largest says what is certainly not among the K best, and the lanes' tiles that have something above it, little more than K of them, are looked at
// again, element by element, for the piece's list.  A second launch joins the pieces of a prompt's rows.  Memory bounds the pass over large calls (512
// rows of 131072 bf16: 27 of the launch's 30 us for 134 MB, 25 without the exponentials), latency the rest: the list takes a block 3 us, the
// join 4 to 6 for up to eight beams.  An element is a key: its
// value in the order of unsigned numbers, above the complement of its index, so that of equal values the first is the larger key; 0
// is no element.
constexpr int kWaves = 4;
constexpr int kTileElems = 2048;     // of a wave: 32 elements a lane
constexpr int kMostTiles = 16;       // of a wave
constexpr int kLooks = 4;
constexpr float kLeast = -3.402823466e38f;   // the lowest finite value

struct PieceStats { float at; double sum; };   // sum of exp(x - at)

__device__ __forceinline__ u64 key_of(float x, uint32_t at) {
  const uint32_t b = __float_as_uint(x + 0.f);   // -0 is 0
  return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | ~at;
}
__device__ __forceinline__ float value_of(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// Bitonic sorting of 64 keys, one a lane, in registers: a step takes the key of the lane J away, by moves inside 16 lanes or a
// swap of 16 or 32, and keeps the larger of the two in the lanes of a mask that is known in advance.  Nine instructions a step; through
// the LDS crossbar a sort takes 1.3 us, so 0.35.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, false); }
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kXor3 = 0x1b, kXor7 = 0x141, kXor8 = 0x128, kXor15 = 0x140;
template <int J>
__device__ __forceinline__ uint32_t lane_across(uint32_t x) {
  if constexpr (J == 1) return moved<kXor1>(x);
  else if constexpr (J == 2) return moved<kXor2>(x);
  else if constexpr (J == 4) return moved<kXor3>(moved<kXor7>(x));
  else return moved<kXor8>(x);
}
struct Pair { u64 a, b; };   // the keys of two lanes: J = 16, 32: the same pair in both, the lower lane's first
template <int J>
__device__ __forceinline__ Pair pair_across(u64 key) {
  const uint32_t lo = (uint32_t)key, hi = (uint32_t)(key >> 32);
  if constexpr (J == 16) {
    const auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    return {(u64)h[0] << 32 | l[0], (u64)h[1] << 32 | l[1]};
  } else if constexpr (J == 32) {
    const auto l = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return {(u64)h[0] << 32 | l[0], (u64)h[1] << 32 | l[1]};
  } else {
    return {key, (u64)lane_across<J>(hi) << 32 | lane_across<J>(lo)};
  }
}
// The lanes that keep the larger key in the step of distance j in runs of k lanes.
constexpr u64 larger_lanes(int k, int j) {
  u64 m = 0;
  for (int l = 0; l < 64; ++l)
    if (((l & k) == 0) == ((l & j) == 0)) m |= 1ull << l;
  return m;
}
template <int K, int J>
__device__ __forceinline__ u64 run_merged(u64 key) {
  const Pair p = pair_across<J>(key);
  key = __builtin_amdgcn_inverse_ballot_w64(__builtin_amdgcn_ballot_w64(p.a > p.b) ^ ~larger_lanes(K, J)) ? p.a : p.b;
  if constexpr (J > 1) return run_merged<K, J / 2>(key);
  else return key;
}
// in descending order
__device__ __forceinline__ u64 sorted(u64 key) {
  key = run_merged<2, 1>(key);
  key = run_merged<4, 2>(key);
  key = run_merged<8, 4>(key);
  key = run_merged<16, 8>(key);
  key = run_merged<32, 16>(key);
  return run_merged<64, 32>(key);
}
// the largest 64 of two such lists
__device__ __forceinline__ u64 joined(u64 list, u64 more) {
  const uint32_t lo = moved<kXor15>((uint32_t)more), hi = moved<kXor15>((uint32_t)(more >> 32));
  const Pair p = pair_across<16>((u64)hi << 32 | lo);
  more = __builtin_amdgcn_inverse_ballot_w64(0x0000ffff0000ffffull) ? p.b : p.a;
  const Pair q = pair_across<32>(more);
  more = __builtin_amdgcn_inverse_ballot_w64(0x00000000ffffffffull) ? q.b : q.a;   // the other list backwards
  return run_merged<64, 32>(list > more ? list : more);
}
__device__ __forceinline__ u64 key_at(u64 key, int lane) {   // (the same lane for all)
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)key, lane);
}

__device__ __forceinline__ void wave_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's 64 largest keys of all that it is given (of which K are wanted), in descending order, one a lane; keys wait in LDS (128 places) until there
// are enough of them for the registers' sort.
struct Best {
  u64 *buffer;
  u64 list, least;   // least: keys up to this are not among the K best, or are in the list
  int n;             // keys that wait

  __device__ __forceinline__ void flush(int K, int lane) {   // the last (up to) 64 of them
    const int from = max(n - 64, 0);
    wave_lds();
    const u64 more = from + lane < n ? buffer[from + lane] : 0;
    wave_lds();
    n = from;
    list = joined(list, sorted(more));
    const u64 last = key_at(list, K - 1);
    least = last > least ? last : least;
  }
  __device__ __forceinline__ void offer(u64 key, bool take, int K, int lane) {
    const u64 m = __ballot(take);
    if (take) buffer[n + __popcll(m & ((1ull << lane) - 1))] = key;
    n += __popcll(m);
    if (n >= 64) flush(K, lane);
  }
};

// Joins the sums of all lanes, in an order that does not depend on the values.
template <int J>
__device__ __forceinline__ void join_step(float &t) { t = fmaxf(t, __uint_as_float(lane_across<J>(__float_as_uint(t)))); }
template <int J>
__device__ __forceinline__ void join_step(double &x) {
  const u64 b = (u64)__double_as_longlong(x);
  x += __longlong_as_double((long long)((u64)lane_across<J>((uint32_t)(b >> 32)) << 32 | lane_across<J>((uint32_t)b)));
}
// unit: the terms are exp(unit) larger than those of exp(x - at).
__device__ __forceinline__ void join_sums(float &at, double &sum, double unit = 0) {
  float t = at;
  join_step<1>(t);
  join_step<2>(t);
  join_step<4>(t);
  join_step<8>(t);
  LanePair p = pair16(t);
  p = pair32(fmaxf(p.a, p.b));
  t = fmaxf(p.a, p.b);
  sum = sum != 0 ? sum * exp((double)at - (double)t - unit) : 0.0;
  join_step<1>(sum);
  join_step<2>(sum);
  join_step<4>(sum);
  join_step<8>(sum);
  sum = add_across<32>(add_across<16>(sum));
  at = t;
}

// A value that at least K of the block's lanes' best are not below, in the order of keys, to its upper 16 bits (all of a bf16's): by bisection,
// four compares and scalar instructions a bit.  0: fewer than K lanes have a finite one.
__device__ __forceinline__ uint32_t kth_of_lanes(const float *best, int lane, int K) {
  uint32_t mine[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float x = best[w * 64 + lane];
    mine[w] = x >= kLeast ? (uint32_t)(key_of(x, 0) >> 32) : 0u;
  }
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t more = t | 1u << bit;
    int n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n += __popcll(__builtin_amdgcn_ballot_w64(mine[w] >= more));
    if (n >= K) t = more;
  }
  return t;
}

// The largest of three, as the instruction itself: the library function first brings operands into canonical form.  (NaN are left out.)
__device__ __forceinline__ float larger(float a, float b, float c) { float r; asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c)); return r; }

// A lane's 32 elements of a tile are 16-byte chunks 64 apart.  Rows start anywhere (the loads are not aligned), and are read once but
// for little (non-temporal loads: 512 rows of 131072 bf16 30.7 -> 29.7 us).  A chunk that ends behind the
// row's end is the row's last 16 bytes, of which what the chunk before it has counts as -inf.
template <int DT>
struct Tile {
  using E = Elem<DT>;
  static constexpr int VEC = E::VEC, CHUNKS = 32 / VEC;
  u32x4 raw[CHUNKS];

  static __device__ __forceinline__ int begin(int tile, int i, int lane) { return tile * kTileElems + (i * 64 + lane) * VEC; }
  static __device__ __forceinline__ int shifted(int V, int e) { return min(e, V - VEC); }
  typedef uint32_t Chunk __attribute__((ext_vector_type(4), aligned(2)));
  __device__ __forceinline__ void load(const char *row, int V, int tile, int lane) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) raw[i] = __builtin_nontemporal_load((const Chunk *)(row + (int64_t)shifted(V, begin(tile, i, lane)) * E::EB));
  }
  // V < VEC: what the shifted chunk has of the row, whose other elements count as -inf anyway
  __device__ __forceinline__ void load_short(const char *row, int V) {
    typename E::Bits b[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) b[j] = ((const typename E::Bits *)row)[max(j - (VEC - V), 0)];
    __builtin_memcpy(&raw[0], b, 16);
#pragma unroll
    for (int i = 1; i < CHUNKS; ++i) raw[i] = raw[0];
  }
  __device__ __forceinline__ void values(int V, int tile, int lane, float (&x)[32]) const {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) E::unpack(raw[i], (float (&)[VEC])x[i * VEC]);
    if ((tile + 1) * kTileElems > V) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int e = begin(tile, i, lane), lost = e - shifted(V, e);
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[i * VEC + j] = j < lost ? -INFINITY : x[i * VEC + j];
      }
    }
  }
};

// The sum's terms are 2^(x L - c), L = log2 e in 32 bits and c the whole number next to at L, for a value `at` of the lane that is at most
// kAbove below its largest element: a change of `at` multiplies the sum by a power of two, which is exact.  A term's exponent is rounded once
// (2^-24 (|x - at| + 0.35) of the term), L is off by 0.23 2^-24, 2^y by 2^-23, and three sums of 2^-24 follow before 64 bits.  The mean of
// |x - at| under the terms' own weights is at most kAbove and the logarithm of a lane's 512 elements (the largest element's distance to the mean
// is an entropy's part): 2^-24 (1.23 (2 + 6.3) + 5.4) = 2^-24 15.6.  Exponents in two parts, whole and rest, would leave half of that for four
// more instructions an element (512 rows of 131072 bf16: 30 -> 34 us).  Where x L leaves no place for a fraction (values beyond 2^20, and
// lanes that have seen nothing but -inf), x - at, which is exact for what counts, takes the place of x, and c is 0.  NaN and +inf make the sum NaN.
constexpr float kLog2e = 0x1.715476p0f, kAbove = 2.f;
constexpr double kLn2 = 0x1.62e42fefa39efp-1;
__device__ __forceinline__ bool is_far(float at) { return !(fabsf(at) <= 0x1p20f); }
__device__ __forceinline__ float whole_of(float at) { return is_far(at) ? 0.f : rintf(at * kLog2e); }
__device__ __forceinline__ double unit_of(float at) { return is_far(at) ? (double)at * (double)kLog2e : (double)whole_of(at); }   // terms are 2^(x L - this)

template <int DT>
__global__ __launch_bounds__(kWaves * 64, DT == THK_F32 ? 3 : 4) void k_beam_pieces(BeamArgs a, int pieces, int tiles_each) {
  using T = Tile<DT>;
  constexpr int EB = Elem<DT>::EB, VEC = T::VEC;
  __shared__ float tile_best[kWaves][kMostTiles][64];
  __shared__ float lane_best[kWaves * 64];
  __shared__ uint16_t looks[kWaves][kMostTiles * 64];         // lanes' tiles to be looked at again
  __shared__ u64 waiting[kWaves][128];
  __shared__ u64 all_keys[kWaves * 128];
  __shared__ PieceStats stats[kWaves];
  __shared__ int n_keys;
  const int64_t row = blockIdx.x / (unsigned)pieces;
  const int piece = (int)(blockIdx.x - row * pieces), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const char *const x_row = (const char *)a.logits + row * a.ld * EB;
  const int first = (piece * kWaves + wave) * tiles_each, last = min(first + tiles_each, (a.V + kTileElems - 1) / kTileElems);
  const int end = a.done != nullptr ? a.done[row] : 0;
  const float before = a.scores[row];
  T next;
  if (a.V < VEC) next.load_short(x_row, a.V);
  else if (first < last) next.load(x_row, a.V, first, lane);
  if (end != 0 || !(fabsf(before) < INFINITY)) return;
  if (threadIdx.x == 0) n_keys = 0;

  float at = kLeast, c = 0, best = -INFINITY;
  double sum = 0;
  for (int tile = first; tile < last; ++tile) {
    float x[32];
    const T now = next;
    if (tile + 1 < last) next.load(x_row, a.V, tile + 1, lane);
    now.values(a.V, tile, lane, x);
    float most = larger(x[0], x[1], x[2]);
#pragma unroll
    for (int i = 3; i < 31; i += 2) most = larger(most, x[i], x[i + 1]);
    most = larger(most, x[31], x[31]);
    best = larger(best, most, most);
    tile_best[wave][tile - first][lane] = most;
    if (__ballot(most - at > kAbove) != 0) {
      const float to = most - at > kAbove ? most : at, c_to = whole_of(to);
      if (sum != 0 && to > at && (is_far(at) || is_far(to))) sum *= exp2(unit_of(at) - unit_of(to));
      else if (to > at) sum = ldexp(sum, (int)(c - c_to));
      at = to;
      c = c_to;
    }
    if (__ballot(is_far(at)) != 0) {
      const float off = is_far(at) ? at : 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] -= off;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = fmaf(x[i], kLog2e, -c);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(x[8 * g + j]);
      sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    }
  }
  lane_best[threadIdx.x] = best;
  join_sums(at, sum, kLn2 * ((double)at * (double)kLog2e - unit_of(at)));
  if (lane == 0) stats[wave] = {at, sum};
  __syncthreads();

  // the list
  const uint32_t kth = kth_of_lanes(lane_best, lane, a.K);
  Best best_keys = {waiting[wave], 0, kth != 0 ? ((u64)kth << 32) - 1 : 0, 0};
  const float least_value = kth != 0 ? value_of((u64)kth << 32) : kLeast;
  int found = 0;
  for (int t0 = 0; t0 < last - first; t0 += 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {      // (kMostTiles is a multiple of four)
      const int t = t0 + u;
      const bool mine = t < last - first && tile_best[wave][t][lane] >= least_value;
      const u64 who = __ballot(mine);
      if (mine) looks[wave][found + __popcll(who & ((1ull << lane) - 1))] = (uint16_t)(t << 6 | lane);
      found += __popcll(who);
    }
  }
  wave_lds();
  for (int f0 = 0; f0 < found; f0 += 2 * kLooks) {      // two lanes' elements at a time, one a lane, their loads under way together
    float y[kLooks];
    int where[kLooks];
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const int f = f0 + 2 * u + (lane >> 5), i = lane & 31, look = looks[wave][min(f, found - 1)];
      const int e = T::begin(first + (look >> 6), i / VEC, look & 63), from = T::shifted(a.V, e), j = i % VEC;
      where[u] = f < found && j >= e - from ? from + j : -1;
      y[u] = Elem<DT>::load1(x_row, max(where[u], 0));
    }
#pragma unroll
    for (int u = 0; u < kLooks; ++u) {
      const u64 key = key_of(y[u], (uint32_t)where[u]);
      best_keys.offer(key, where[u] >= 0 && y[u] >= kLeast && y[u] < INFINITY && key > best_keys.least, a.K, lane);
    }
  }
  wave_lds();
#pragma unroll
  for (int part = 0; part < 2; ++part) {   // the waves' keys together
    const u64 key = part == 0 ? (lane < best_keys.n ? best_keys.buffer[lane] : 0) : (lane < a.K ? best_keys.list : 0);
    const u64 m = __ballot(key != 0);
    if (m == 0) continue;
    int base = lane == 0 ? atomicAdd(&n_keys, __popcll(m)) : 0;
    base = __builtin_amdgcn_readfirstlane(base);
    if (key != 0) all_keys[base + __popcll(m & ((1ull << lane) - 1))] = key;
  }
  __syncthreads();
  if (wave == 1) {
    PieceStats s = lane < kWaves ? stats[lane] : PieceStats{kLeast, 0.0};
    join_sums(s.at, s.sum);
    if (lane == 0) ((PieceStats *)a.ws)[blockIdx.x] = s;
  }
  if (wave != 0) return;
  const int total = n_keys;
  u64 list = sorted(lane < total ? all_keys[lane] : 0);
  for (int i = 64; i < total; i += 64) list = joined(list, sorted(i + lane < total ? all_keys[i + lane] : 0));
  u64 *const out = (u64 *)((PieceStats *)a.ws + (int64_t)a.B * a.W * pieces) + (int64_t)blockIdx.x * a.K;
  if (lane < a.K) out[lane] = list;
}


// A block of eight waves, or sixteen where that spares them rows (32 beams, the best 64 of 149134 tokens: 51 -> 41 us for the call of then), joins a
// prompt: a wave for each row joins its pieces' lists and sums, then the rows' candidates are ranked by counting.  Pieces and join: one prompt of 32 beams,
// the best 64 of 149134 bf16, 12.3 + 20.2 us, four prompts 17.3 + 15.9 (fp32: 13.0 + 20.0, 21.5 + 15.8); 16 beams, the best 32, 8.2 + 8.9 and
// 10.6 + 7.6; 8 beams, the best 16, 7.2 + 5.6 and 8.3 + 5.9.  One block sorts and ranks for a prompt, which bounds the long lists of many beams.
constexpr int join_waves(int W) { return W <= 8 ? 8 : 16; }
template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_beam_join(BeamArgs a, int pieces) {
  __shared__ double score[kMostBeams * kMostContinuations];
  __shared__ u64 waiting[WAVES][128];
  __shared__ int at[kMostBeams * kMostContinuations];      // tokens; entry beam * K + place in the beam's list
  __shared__ double live_score[kMostBeams * kMostContinuations];
  __shared__ int live_at[kMostBeams * kMostContinuations];
  __shared__ double kth[kMostBeams];
  __shared__ int ended[kMostBeams];
  __shared__ int n_live;
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const PieceStats *const stats = (const PieceStats *)a.ws;
  if (tid == 0) n_live = 0;
  const int count = pieces * a.K;
  for (int w = wave; w < a.W; w += WAVES) {
    const int64_t row = b * a.W + w;
    const float before = a.scores[row];
    const bool end = a.done != nullptr && a.done[row] != 0;
    // (asked for before it is known whether they are there)
    const u64 *const keys = (const u64 *)(stats + (int64_t)a.B * a.W * pieces) + row * count;
    u64 more = lane < count ? keys[lane] : 0;
    PieceStats x = lane < pieces ? stats[row * pieces + lane] : PieceStats{kLeast, 0.0};
    double s = -INFINITY;
    int token = 0;
    if (!(fabsf(before) < INFINITY)) {
    } else if (end) {
      if (lane == 0) s = before;
      token = a.eos;
    } else {
      for (int p = lane + 64; p < pieces; p += 64) {
        const PieceStats y = stats[row * pieces + p];
        const float to = fmaxf(x.at, y.at);
        x.sum = (x.sum != 0 ? x.sum * exp((double)x.at - (double)to) : 0) + (y.sum != 0 ? y.sum * exp((double)y.at - (double)to) : 0);
        x.at = to;
      }
      Best best_keys = {waiting[wave], sorted(more), 0, 0};
      best_keys.least = key_at(best_keys.list, a.K - 1);
      for (int i = 64; i < count; i += 4 * 64) {
        u64 four[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) four[u] = keys[min(i + u * 64 + lane, count - 1)];   // (all under way at once)
#pragma unroll
        for (int u = 0; u < 4; ++u) best_keys.offer(four[u], i + u * 64 + lane < count && four[u] > best_keys.least, a.K, lane);
      }
      if (best_keys.n > 0) best_keys.flush(a.K, lane);
      const u64 list = best_keys.list;
      join_sums(x.at, x.sum);
      if (list != 0 && lane < a.K) {   // (a sum that is NaN leaves no score)
        s = (double)before + (((double)value_of(list) - (double)x.at) - log(x.sum));
        token = (int)~(uint32_t)list;
        if (!(fabs(s) < INFINITY)) s = -INFINITY;
      }
    }
    if (lane < a.K) {
      score[w * a.K + lane] = s;
      at[w * a.K + lane] = token;
      if (lane == a.K - 1) kth[w] = s;
    }
    if (lane == 0) ended[w] = end;
  }
  __syncthreads();
  // what is below the K-th of one row is not among the K best of all
  double floor = -INFINITY;
  for (int w = 0; w < a.W; ++w) floor = fmax(floor, kth[w]);
  for (int i = tid; i < a.W * a.K; i += WAVES * 64)
    if (score[i] > -INFINITY && score[i] >= floor) {
      const int to = atomicAdd(&n_live, 1);
      live_score[to] = score[i];
      live_at[to] = i;      // (equal scores: by the beam, then by its list, which is by logits and then tokens)
    }
  __syncthreads();
  const int n = n_live;
  // A wave ranks four candidates at a time, a lane of it compares them with its part of all (8 x 16 candidates a prompt, 64 prompts: 5.8 us;
  // a candidate a lane, against all: 8.1).
  for (int i0 = wave * 4; i0 < n; i0 += WAVES * 4) {
    double s[4];
    int mine[4], rank[4] = {};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      s[u] = live_score[min(i0 + u, n - 1)];
      mine[u] = live_at[min(i0 + u, n - 1)];
    }
    for (int j0 = 0; j0 < n; j0 += 64) {
      const int j = min(j0 + lane, n - 1), y = live_at[j];
      const double x = j0 + lane < n ? live_score[j] : -INFINITY;
#pragma unroll
      for (int u = 0; u < 4; ++u) rank[u] += __popcll(__ballot(x > s[u] || (x == s[u] && y < mine[u])));
    }
    int r = rank[0], i = mine[0];
    double score_of = s[0];
#pragma unroll
    for (int u = 1; u < 4; ++u) {
      r = lane == u ? rank[u] : r;
      i = lane == u ? mine[u] : i;
      score_of = lane == u ? s[u] : score_of;
    }
    if (lane >= min(4, n - i0) || r >= a.K) continue;
    const int64_t out = b * a.K + r;
    const int w = i / a.K, token = at[i];
    a.parent[out] = w;
    a.token[out] = token;
    a.score_out[out] = (float)score_of;
    if (a.done_out != nullptr) a.done_out[out] = token == a.eos || ended[w] != 0;
  }
  for (int k = n + tid; k < a.K; k += WAVES * 64) {
    const int64_t out = b * a.K + k;
    a.parent[out] = -1;
    a.token[out] = -1;
    a.score_out[out] = -INFINITY;
    if (a.done_out != nullptr) a.done_out[out] = 0;
  }
}

// ---- caches that follow -------------------------------------------------------------------
// A thread has one place of 16 bytes in the keys' (or values') tails of all beams of a prompt: it reads the parents' before it writes any, so
// that beams may go on from each other in place.  (Parents and row counts are the same for a block: they go through the scalar unit.)  Memory bounds it:
// 64 beams of 8 layers and 8 heads, 190 MB read and written, 36 us, 5.2 TB/s, for prompts of 8 beams; of 16 beams 48 us, of 32 47 (five and three
// waves a SIMD instead of eight, for a thread's W places).
template <int DT, int W>
__global__ __launch_bounds__(256) void k_reorder_tails(ReorderArgs a, int blocks) {
  constexpr int CPR = kD * Elem<DT>::EB / 16;
  __shared__ int from[W], rows[W], tail[W], most;
  const int64_t g2 = blockIdx.x / (unsigned)blocks, g = g2 >> 1;    // (layer, prompt, head), keys or values
  const int64_t lp = g / a.N_kv, h = g - lp * a.N_kv, p = lp % a.prompts;
  const int tid = threadIdx.x;
  if (tid == 0) most = 0;
  int par = -1;
  if (tid < W) {
    if (tid < a.W) {
      par = a.parent[p * a.ld_parent + tid];
      tail[tid] = a.s_tail[p * a.W + tid];
    }
    rows[tid] = from[tid] = 0;
  }
  __syncthreads();
  if (tid < a.W && par >= 0 && par < a.W && par != tid) {
    const int n = min(tail[par], a.cap);
    from[tid] = par;
    rows[tid] = n;
    if (n > 0) atomicMax(&most, n);
  }
  __syncthreads();
  const int64_t stride = (int64_t)a.N_kv * a.cap * CPR;
  u32x4 *const x0 = (u32x4 *)(g2 & 1 ? a.v_tail : a.k_tail) + (lp * a.W * a.N_kv + h) * a.cap * CPR;
  int n[W];
  int64_t at[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    n[j] = __builtin_amdgcn_readfirstlane(rows[j]);
    at[j] = (int64_t)__builtin_amdgcn_readfirstlane(from[j]) * stride;
  }
  const int64_t last = (int64_t)most * CPR;
  for (int64_t c = (blockIdx.x - g2 * blocks) * 256 + tid; c < last; c += (int64_t)blocks * 256) {
    const int row = (int)(c / CPR);
    u32x4 *const x = x0 + c;
    u32x4 v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = x[row < n[j] ? at[j] : at[0]];   // (any of the thread's own places where there is nothing to take)
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (row < n[j]) x[j * stride] = v[j];
  }
}

// A prompt's table rows and counts, likewise: a thread has one entry of all beams.  Latency: two trips, 3.1 us for 4 beams, 5.0 for 8 of 16 pages; 7.6 for 16, 12.3
// for 32, each entry's loads and stores by one thread.
template <int W>
__global__ __launch_bounds__(256) void k_reorder_pages(ReorderArgs a) {
  __shared__ int from[W], mine[W], keep[W], old_held[W], old_pages[W], old_tail[W], most;
  const int64_t p = blockIdx.x;
  const int tid = threadIdx.x;
  if (tid == 0) most = 0;
  if (tid < W) {
    from[tid] = -1;
    mine[tid] = keep[tid] = 0;     // entries given up, entries taken over
  }
  if (tid < a.W) {
    const int64_t b = p * a.W + tid;
    const int par = a.parent[p * a.ld_parent + tid];
    from[tid] = par >= 0 && par < a.W && par != tid ? par : -1;
    old_held[tid] = a.max_pages > 0 ? min(max(a.held[b], 0), a.max_pages) : 0;
    old_pages[tid] = a.s_pages != nullptr ? a.s_pages[b] : 0;
    old_tail[tid] = a.s_tail != nullptr ? a.s_tail[b] : 0;
  }
  __syncthreads();
  if (tid < a.W) {
    const int64_t b = p * a.W + tid;
    const int f = from[tid];
    if (f >= 0) {
      mine[tid] = old_held[tid];
      keep[tid] = (int)min((int64_t)old_held[f], ((int64_t)max(old_pages[f], 0) + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift);
      atomicMax(&most, max(mine[tid], keep[tid]));
      if (a.max_pages > 0) a.held[b] = keep[tid];
      if (a.s_pages != nullptr) a.s_pages[b] = old_pages[f];
      if (a.s_tail != nullptr) a.s_tail[b] = old_tail[f];
    }
  }
  __syncthreads();
  const int last = most;
  int32_t *const table = a.table + p * a.W * a.max_pages;
  for (int e = tid; e < last; e += 256) {
    int old[W], now[W];   // (all loads under way at once)
#pragma unroll
    for (int j = 0; j < W; ++j) {
      old[j] = table[(int64_t)min(j, a.W - 1) * a.max_pages + e];
      now[j] = table[(int64_t)max(from[j], 0) * a.max_pages + e];
    }
#pragma unroll
    for (int j = 0; j < W; ++j) {
      old[j] = e < mine[j] ? old[j] : -1;
      now[j] = e < keep[j] ? now[j] : -1;
    }
#pragma unroll
    for (int j = 0; j < W; ++j) {
      if (e >= max(mine[j], keep[j])) continue;
      if (now[j] != old[j]) {
        if (old[j] >= 0 && old[j] < a.n_pages) atomicAdd(a.refs + old[j], -1);
        if (now[j] >= 0 && now[j] < a.n_pages) atomicAdd(a.refs + now[j], 1);
      }
      table[(int64_t)j * a.max_pages + e] = now[j];
    }
  }
}

template <class... A>
hipError_t launch(const void *k, int64_t blocks, int threads, hipStream_t st, A... a) {
  void *args[] = {&a...};
  return launch_main_kernel(k, dim3((unsigned)blocks), dim3(threads), args, 0, st);
}

// Into how many pieces a row is cut, by an estimate in half microseconds, fitted to 180 measured calls of 2 to 205 MB (off by a tenth of the time): a tile
// of every wave takes the k blocks of a compute unit 0.5 us (fp32: 1) k and 0.25, the rest 0.9 us k, in as many rounds as there are of
// blocks that fit; the join takes a wave 0.35 us for 64 keys.  512 rows of 131072 bf16: 36.6 us with one piece, 35.8 two, 38.6 four, 44.7
// eight; 184 of 208660: 25.3 two, 24.1 four, 26.3 five, 28.1 six; 76 of 106494 fp32: 17.1 two, 15.4 three, 16.0 seven; 4 of 32768
// bf16: 10.4 four, 10.8 two, 12.1 one.
struct BeamPlan { int pieces, tiles_each; };
BeamPlan beam_plan(int dtype, const BeamArgs &a) {
  const int64_t tiles = ((int64_t)a.V + kTileElems - 1) / kTileElems, rows = (int64_t)a.B * a.W;
  const int64_t fit = dtype == THK_F32 ? 3 : 4, tile = dtype == THK_F32 ? 2 : 1;   // blocks of a compute unit
  BeamPlan best{};
  double least = 0;
  for (int64_t each = 1; each <= kMostTiles; ++each) {
    const int64_t pieces = (tiles + each * kWaves - 1) / (each * kWaves);
    if (pieces == best.pieces) continue;   // (as many with fewer tiles)
    auto round = [&](int64_t k) { return k == 0 ? 0. : each * (tile * k + 0.5) + 1.8 * k; };
    const int64_t k = (rows * pieces + kCUs - 1) / kCUs, of_a_wave = (a.W + join_waves(a.W) - 1) / join_waves(a.W);
    const double t = k / fit * round(fit) + round(k % fit) + 0.7 / 64 * pieces * a.K * of_a_wave;
    if (best.pieces == 0 || t < least) {
      least = t;
      best = {(int)pieces, (int)each};
    }
  }
  return best;
}

template <int W>
hipError_t reorder(int dtype, const ReorderArgs &a, hipStream_t st) {
  if (a.cap > 0) {
    const int64_t groups = (int64_t)2 * a.L * a.prompts * a.N_kv, most = (a.cap * (int64_t)(dtype == THK_F32 ? 32 : 16) + 255) / 256;
    const int blocks = (int)std::min(most, std::max<int64_t>(1, 16 * kCUs / groups));
    const hipError_t e = launch(dtype == THK_F32 ? (const void *)k_reorder_tails<THK_F32, W> : (const void *)k_reorder_tails<THK_BF16, W>,
                                groups * blocks, 256, st, a, blocks);
    if (e != hipSuccess) return e;
  }
  return launch((const void *)k_reorder_pages<W>, a.prompts, 256, st, a);
}

}  // namespace

size_t beam_ws_bytes(int dtype, const BeamArgs &a) {
  const int64_t pieces = beam_plan(dtype, a).pieces, blocks = (int64_t)a.B * a.W * pieces;
  return blocks * kWaves * 64 > 0xffffffffll || (int64_t)a.B * 1024 > 0xffffffffll ? 0 : (size_t)blocks * (sizeof(PieceStats) + a.K * sizeof(u64));
}

hipError_t launch_beam_select(int dtype, const BeamArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  const BeamPlan p = beam_plan(dtype, a);
  const hipError_t e = launch(dtype == THK_F32 ? (const void *)k_beam_pieces<THK_F32> : (const void *)k_beam_pieces<THK_BF16>, (int64_t)a.B * a.W * p.pieces,
                              kWaves * 64, st, a, p.pieces, p.tiles_each);
  if (e != hipSuccess) return e;
  return launch(join_waves(a.W) == 8 ? (const void *)k_beam_join<8> : (const void *)k_beam_join<16>, a.B, join_waves(a.W) * 64, st, a, p.pieces);
}

hipError_t launch_reorder(int dtype, const ReorderArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  return a.W <= 4 ? reorder<4>(dtype, a, st) : a.W <= 8 ? reorder<8>(dtype, a, st) : a.W <= 16 ? reorder<16>(dtype, a, st) : reorder<32>(dtype, a, st);
}

}  // namespace thk
