// Attention of one new token over a paged cache and a tail: the kernel, for both element types and all page formats.
//
//   z_r = scale * sum_t q_t k_rt,  out = sum_r p_r v_r / sum_r p_r,  p_r = 2^(z_r - m)
// With codes, k_rt = m_t + s_t c_rt (a group's scale and minimum, t a channel of the tile), so
//   z_r = scale * ( sum_t q_t m_t  +  sum_t (q_t s_t) c_rt ):
// the query takes the scales, once per tile, and the codes enter the matrix cores as the whole numbers they are, which
// bf16 holds exactly.  Values likewise: sum_r p_r v_rc = sum_r p_r m_r + sum_r (p_r s_r) c_rc.  What is not exact in bf16 --
// the scaled query and the scaled probabilities -- enters as a sum of bf16 terms: two for bf16 tensors (2^-17 of the value),
// three for fp32 ones (2^-25).  Two cost a bf16 output nothing but, now and then, the choice between two neighbours: of 4-bit
// codes, 640 heads over up to 8192 rows, 1.8 % of the outputs are not the nearest bf16 number but the next one (fp32 arithmetic
// throughout: 0.05 %), of 8-bit codes 0.7 %, of elements 0.2 to 0.4 %; the error against 64 bits, 1.7e-3, is that of the rounding.
// Of a code c an operand holds something more, which is taken out again with the minimum: 4-bit codes of bf16 tensors are used
// as 16 + c, whose bits are the code in the mantissa of 16 (one shift and one mask for two of them); those of fp32 tensors as c
// less half the range, a signed byte, which keeps the two sums that make up a logit small and with them what their rounding
// costs (8 bits, 2048 rows: 1.5e-6 of the result with plain codes, 2.4e-7 so).  8-bit codes of bf16 tensors are plain, an
// instruction less for each word: 1.5e-6 is nothing beside the output's rounding.
//
// A wave takes a tile of 64 rows at a time.  S^T = K q^T: A = 16 rows x 32 channels of keys, B = 32 channels x 16 query
// heads, so lane (m, h) = (lane % 16, lane / 16) ends up with the logits of head m for rows 16 j + 4 h + i.  out^T = V^T P^T:
// B = 32 rows x 16 heads wants from lane (m, h) eight rows of head m, and the groups of the values are made of just the
// rows the lane holds: the probabilities go from one product into the other in the lane's own registers.
//
// What bounds the kernel over codes is the vector unit's work per tile -- scales, softmax, terms -- which costs the same for
// one query head as for sixteen.  So a wave takes CL tiles at once where few heads share a KV head: of the sixteen columns,
// 16 / CL are heads of the first tile, the next 16 / CL the same heads of the second, and so on.  A lane scales its query by
// its own tile's scales, keeps the logits of its own tile, and scales the probabilities by its own tile's scales, all for CL
// tiles at the price of one; the matrix cores multiply every tile with all columns, the columns of other tiles being left out
// by a select (logits) or a mask (probabilities).  The CL columns of a head are states of their own until the end.
// Columns past the last head are zeros.
//
// Measured (kernel alone; a kernel that only reads the bytes reaches 7.1 TB/s): bf16 elements, 8 units of four heads x 131072 rows
// 62 us, 6.5 TB/s; 4-bit codes, 640 units of one head, up to 8192 rows 79 us, 4.5 TB/s (vector unit busy half of the time, matrix
// cores a fifth), 256 units of four heads x 32768 rows 146 us, 6.3 TB/s, and up to 224 when such calls follow one another for some
// ms and the card lowers its clock; 8-bit codes, 64 units of eight heads, up to 8191 rows 22 us, 3.5 TB/s: pieces of some 24 tiles,
// three steps of a wave, whose ramp is as long as they are.
// 8 units x 1000 rows 5.4 us: launch, three trips to memory one after another (lengths, table, tiles), the states' exchange.
#pragma once
#include "thk_paged.h"

namespace thk {
namespace paged {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// An address of device memory where the compiler does not see that it is one (it would load through the path that may also reach
// LDS, whose loads are waited for all at once).
#define THK_GLOBAL __attribute__((address_space(1)))
typedef THK_GLOBAL char *GlobalPtr;
__device__ __forceinline__ GlobalPtr as_global(const void *p) { return (GlobalPtr)(uintptr_t)p; }

// Eight floats as NT bf16 terms that add up to them: each term is what the ones in front left over.
template <int NT>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8 (&t)[NT]) {
  f32x2 r[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) r[p] = f32x2{x[2 * p], x[2 * p + 1]};
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const bf16x2 c = __builtin_convertvector(r[p], bf16x2);
      t[n][2 * p] = c[0];
      t[n][2 * p + 1] = c[1];
      if (n + 1 < NT) r[p] -= __builtin_convertvector(c, f32x2);
    }
}

template <int DT, int BITS>
struct Format {
  static constexpr bool kCodes = BITS != 0;
  static constexpr bool kFp32 = DT == THK_F32 && !kCodes;     // products on the fp32 matrix instructions
  static constexpr int UB = kCodes ? BITS : 8 * Elem<DT>::EB;   // bytes of a unit
  static constexpr int NC = UB / 4;                           // 16-byte cells of a lane in a group
  static constexpr int NTK = !kCodes ? 1 : DT == THK_F32 ? 3 : 2;   // terms of the (scaled) query
  static constexpr int NTV = DT == THK_F32 ? 3 : 2;                 // terms of the (scaled) probabilities
  // an operand is kTimes * code + kBias
  static constexpr bool kMantissa = BITS == 4 && DT == THK_BF16;
  static constexpr bool kPlain = BITS == 8 && DT == THK_BF16;
  static constexpr float kTimes = BITS == 4 && !kMantissa ? 16.f : 1.f;
  static constexpr float kBias = kMantissa ? 16.f : kPlain ? 0.f : -128.f;
};

// Signed bytes A and B of x as two bf16 numbers: whole numbers below 256 in size have all their bits in a float's upper half.
template <int A, int B>
__device__ __forceinline__ uint32_t byte_pair(uint32_t x) {
  return __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(x >> (8 * B))), __float_as_uint((float)(int8_t)(x >> (8 * A))), 0x07060302u);
}

// ... unsigned ones.
template <int A, int B>
__device__ __forceinline__ uint32_t code_pair(uint32_t x) {
  return __builtin_amdgcn_perm(__float_as_uint((float)((x >> (8 * B)) & 255u)), __float_as_uint((float)((x >> (8 * A)) & 255u)), 0x07060302u);
}

// Constants of the 4-bit form, in vector registers: an instruction takes one scalar operand only.
struct Mantissa {
  uint32_t mask = 0x00780078u, one = 0x41804180u;
  __device__ __forceinline__ Mantissa() { asm("" : "+v"(mask), "+v"(one)); }
};

// Unit j of a lane's cells as an operand of eight.
template <int DT, int BITS>
__device__ __forceinline__ bf16x8 operand(const u32x4 (&w)[Format<DT, BITS>::NC], int j, const Mantissa &c) {
  u32x4 u;
  if constexpr (Format<DT, BITS>::kMantissa) {
    const uint32_t x = w[0][j];
    u[0] = ((x << 3) & c.mask) | c.one;
    u[1] = ((x >> 1) & c.mask) | c.one;
    u[2] = ((x >> 5) & c.mask) | c.one;
    u[3] = ((x >> 9) & c.mask) | c.one;
  } else if constexpr (BITS == 4) {   // a code in the upper half of a byte: 16 c - 128 as a signed byte
    const uint32_t even = ((w[0][j] << 4) & 0xf0f0f0f0u) ^ 0x80808080u, odd = (w[0][j] & 0xf0f0f0f0u) ^ 0x80808080u;
    u[0] = byte_pair<0, 2>(even);
    u[1] = byte_pair<0, 2>(odd);
    u[2] = byte_pair<1, 3>(even);
    u[3] = byte_pair<1, 3>(odd);
  } else if constexpr (Format<DT, BITS>::kPlain) {
    const uint32_t lo = w[j >> 1][2 * (j & 1)], hi = w[j >> 1][2 * (j & 1) + 1];
    u[0] = code_pair<0, 1>(lo);
    u[1] = code_pair<2, 3>(lo);
    u[2] = code_pair<0, 1>(hi);
    u[3] = code_pair<2, 3>(hi);
  } else if constexpr (BITS == 8) {
    const uint32_t lo = w[j >> 1][2 * (j & 1)] ^ 0x80808080u, hi = w[j >> 1][2 * (j & 1) + 1] ^ 0x80808080u;
    u[0] = byte_pair<0, 1>(lo);
    u[1] = byte_pair<2, 3>(lo);
    u[2] = byte_pair<0, 1>(hi);
    u[3] = byte_pair<2, 3>(hi);
  } else {
    u = w[j];
  }
  return __builtin_bit_cast(bf16x8, u);
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// The fp32 form of the same product: its k index runs over the four quarters of the wave, so eight instructions take the
// lanes' eight elements one by one.
__device__ __forceinline__ f32x4 mfma16_f32(const float (&a)[8], const float (&b)[8], f32x4 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ float sum_quarters(float x) {
  LanePair p = pair16(x);
  p = pair32(p.a + p.b);
  return p.a + p.b;
}
__device__ __forceinline__ float max_quarters(float x) {
  LanePair p = pair16(x);
  p = pair32(fmaxf(p.a, p.b));
  return fmaxf(p.a, p.b);
}

// scale and minimum of the eight pairs at `par`
template <int DT>
__device__ __forceinline__ void load_pairs(GlobalPtr par, u32x4 (&w)[DT == THK_BF16 ? 2 : 4]) {
#pragma unroll
  for (int i = 0; i < (DT == THK_BF16 ? 2 : 4); ++i) w[i] = ((const THK_GLOBAL u32x4 *)par)[i];
}
template <int DT>
__device__ __forceinline__ void pair_of(const u32x4 (&w)[DT == THK_BF16 ? 2 : 4], int e, float &s, float &lo) {
  if constexpr (DT == THK_BF16) {
    s = __uint_as_float(w[e >> 2][e & 3] << 16);
    lo = __uint_as_float(w[e >> 2][e & 3] & 0xffff0000u);
  } else {
    s = __uint_as_float(w[e >> 1][2 * (e & 1)]);
    lo = __uint_as_float(w[e >> 1][2 * (e & 1) + 1]);
  }
}

// A wave's running softmax, of the lane's column.  acc[4 half + i][r]: channel 64 half + 16 h + 4 r + i.
struct State {
  f32x4 acc[8];
  float off[2];   // this lane's share of sum_r p_r m_r per half of the channels
  float l;        // this lane's share of sum_r p_r
  float m;        // whole number: every change of it scales by an exact power of two
};

// p[j][i] <- 2^(scale z - m) for the logits z of the lane's tile, of which `rows` rows count (none: the column has no tile);
// the state is brought to the new m.
__device__ __forceinline__ void softmax_step(f32x4 (&z)[4], int rows, int h, float scale, State &st) {
  if (__any(rows < kTile)) {
    int left = rows - 4 * h;
    asm("" : "+v"(left));   // (else the sixteen rows' numbers are kept in registers through the loop)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (16 * j + i >= left) z[j][i] = -INFINITY;
      __builtin_amdgcn_sched_barrier(0);   // (sixteen comparisons ahead of their use would take 32 scalar registers)
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, z[j][i]);
  const float m_new = fmaxf(st.m, ceilf(max_quarters(mx) * scale));
  if (__any(m_new > st.m)) {
    const float keep = st.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m - m_new);
#pragma unroll
    for (int i = 0; i < 8; ++i) st.acc[i] *= keep;
    st.off[0] *= keep;
    st.off[1] *= keep;
    st.l *= keep;
    st.m = m_new;
  }
  const float m = st.m == -INFINITY ? 0.f : st.m;   // a column without any row so far: all weights are 0
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      z[j][i] = __builtin_amdgcn_exp2f(fmaf(z[j][i], scale, -m));
      sum += z[j][i];
    }
  st.l += sum;
}

// The lane's eight channels of its head per step of 32 kept channels (zeros past T).
template <int DT>
struct Query {
  float x[8];
  __device__ __forceinline__ float operator[](int e) const { return x[e]; }
  __device__ __forceinline__ void set(int e, float v) { x[e] = v; }
  __device__ __forceinline__ void keep() {}
};
template <>
struct Query<THK_BF16> {
  bf16x8 x;
  __device__ __forceinline__ float operator[](int e) const { return (float)x[e]; }
  __device__ __forceinline__ void set(int e, float v) { x[e] = (__bf16)v; }   // exact: v is an element
  // stays as it is from tile to tile: left to itself the compiler widens it once, in front of the loop, into twice the registers
  __device__ __forceinline__ void keep() {
    u32x4 w = __builtin_bit_cast(u32x4, x);
    asm("" : "+v"(w));
    x = __builtin_bit_cast(bf16x8, w);
  }
};

// CL tiles of pages in a wave's registers: t[x] is the x-th (any of the others again where there is none), `own` the lane's
// own, of which `rows` rows count.  The keys and the two halves of the values (by rows) are loaded on their own, each as soon as
// what was loaded two parts before has been used: two of the three parts are in registers or on their way at any time.
template <int DT, int BITS, int NST, int CL>
struct Tiles {
  using F = Format<DT, BITS>;
  static constexpr int NP = F::kCodes ? (DT == THK_BF16 ? 2 : 4) : 1;
  static constexpr int kPairs = 8 * 2 * Elem<DT>::EB;   // bytes of a group's parameters
  // an instruction waits for the one in front of it in its own sum: so many sums in turn (fewer where the registers are full)
  static constexpr int kInTurn = F::kCodes && NST == 3 && CL * BITS == 16 ? 2 : 4;
  static constexpr int kPastEnd = 1 << 20;
  static_assert(kPastEnd >= kMostTileBytes);
  u32x4 kc[CL][NST][F::NC], kp[F::kCodes ? NST : 1][NP];
  u32x4 vc[CL][4][F::NC], vp[F::kCodes ? 4 : 1][NP];

  // 16 bytes of a tile at a lane's offset and a scalar one, through a resource in scalar registers (read once: not to be
  // cached).  bytes: the tile's, or 0: zeros, and memory is not asked (the lane's offset alone is compared with them: with none
  // every one is past the end, and with the tile's none can be)
  static __device__ __forceinline__ u32x4 load_cell(const char *t, int bytes, int lane_off, int off) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)t, (short)0, bytes, 0x00027000);
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane_off, off, 2));
  }
  __device__ __forceinline__ void load_keys(const char *const (&t)[CL], int bytes, GlobalPtr own, const PagedLayout &lay, int m, int h) {
#pragma unroll
    for (int s = 0; s < NST; ++s) {
      // group 4 s + h; of codes those past the last are what lies behind the keys in the tile, which is finite and meets zeros of the
      // query.  (Elements there need not be finite, nor those of a group that is there: an offset past the tile's end loads zeros.)
      if constexpr (F::kCodes) load_pairs<DT>(own + lay.k_params + s * 4 * kPairs, kp[s]);
      const int at = F::kCodes ? h * 64 * F::UB : 4 * s + h < lay.chunks ? (4 * s + h) * 64 * F::UB : kPastEnd, off = F::kCodes ? s * 256 * F::UB : 0;
#pragma unroll
      for (int x = 0; x < CL; ++x)
#pragma unroll
        for (int k = 0; k < F::NC; ++k) kc[x][s][k] = load_cell(t[x], bytes, at + m * 16 + k * 256, off);
    }
  }
  // (G0, G1: which halves of the rows)
  template <int G0 = 0, int G1 = 2>
  __device__ __forceinline__ void load_values(const char *const (&t)[CL], int bytes, GlobalPtr own, const PagedLayout &lay, int m, int h) {
    const GlobalPtr par = own + (uint32_t)(h * kPairs) + lay.v_params;   // (own has one h already)
#pragma unroll
    for (int gh = 2 * G0; gh < 2 * G1; ++gh) {
      const int grp = (gh >> 1) * 8 + (gh & 1);   // the lane's group, less 2 h
      if constexpr (F::kCodes) load_pairs<DT>(par + grp * kPairs, vp[gh]);
#pragma unroll
      for (int x = 0; x < CL; ++x)
#pragma unroll
        for (int k = 0; k < F::NC; ++k) vc[x][gh][k] = load_cell(t[x], bytes, h * 2 * 64 * F::UB + m * 16 + k * 256, lay.v_codes + grp * 64 * F::UB);
    }
  }

  // Half G of the values past the last of `rows` rows becomes zeros: a weight of zero does not take an infinity or NaN out of a
  // sum.  (Elements only: codes are finite.)
  template <int G>
  __device__ __forceinline__ void drop_values(int rows, int h) {
    if constexpr (!F::kCodes) {
      const int left = rows - 4 * h - 32 * G;
      if constexpr (DT == THK_BF16) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int r = 16 * (w >> 1) + 2 * (w & 1);
          const uint32_t keep = (r < left ? 0xffffu : 0u) | (r + 1 < left ? 0xffff0000u : 0u);
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int k = 0; k < F::NC; ++k) vc[0][2 * G + half][k][w] &= keep;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool keep = 16 * (e >> 2) + (e & 3) < left;
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              u32x4 &x = vc[0][2 * G + half][2 * i + (e >> 2)];
              x[e & 3] = keep ? x[e & 3] : 0u;
            }
        }
      }
    }
  }

  // z: the logits of the lane's tile (less the scale); cls: its place
  __device__ __forceinline__ void logits(const Query<DT> (&q)[NST], int cls, const Mantissa &cst, f32x4 (&z)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (F::kFp32) {
#pragma unroll
      for (int s = 0; s < NST; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(kc[0][s][2 * j + (e >> 2)][e & 3]);
          z[j] = mfma16_f32(x, q[s].x, z[j]);
        }
      return;
    }
    bf16x8 b[NST][F::NTK];
    float off = 0.f;
#pragma unroll
    for (int s = 0; s < NST; ++s) {
      if constexpr (F::kCodes) {
        float qs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float sc, lo;
          pair_of<DT>(kp[s], e, sc, lo);
          off = fmaf(q[s][e], lo, off);
          qs[e] = q[s][e] * (sc * (1.f / F::kTimes));
          if constexpr (!F::kPlain) off = fmaf(qs[e], -F::kBias, off);
        }
        split_terms<F::NTK>(qs, b[s]);
      } else if constexpr (DT == THK_BF16) {
        b[s][0] = q[s].x;
      }
    }
#pragma unroll
    for (int x = 0; x < CL; ++x) {
      // operands are made where they are used, not ahead: they would not fit into the registers
      if constexpr (F::kCodes) __builtin_amdgcn_sched_barrier(0);
      f32x4 zx[4] = {};
#pragma unroll
      for (int s = 0; s < NST; ++s) {
#pragma unroll
        for (int j0 = 0; j0 < 4; j0 += kInTurn) {
          bf16x8 a[kInTurn];
#pragma unroll
          for (int j = 0; j < kInTurn; ++j) a[j] = operand<DT, BITS>(kc[x][s], j0 + j, cst);
#pragma unroll
          for (int n = 0; n < F::NTK; ++n)
#pragma unroll
            for (int j = 0; j < kInTurn; ++j) zx[j0 + j] = mfma16(a[j], b[s][n], zx[j0 + j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) z[j][i] = x == 0 || cls == x ? zx[j][i] : z[j][i];
    }
    if constexpr (F::kCodes) {
      off = sum_quarters(off);
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] += off;
    }
  }

  // the values of half G of the rows with the weights w
  template <int G>
  __device__ __forceinline__ void add_values(const f32x4 (&w)[4], int cls, const Mantissa &cst, State &st) const {
    uint32_t mine[CL];
#pragma unroll
    for (int x = 0; x < CL; ++x) mine[x] = cls == x ? 0xffffffffu : 0u;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      constexpr int g = G;
      const int gh = 2 * g + half;
      if constexpr (F::kCodes) __builtin_amdgcn_sched_barrier(0);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = w[2 * g + (e >> 2)][e & 3];
      if constexpr (F::kFp32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(vc[0][gh][2 * i + (e >> 2)][e & 3]);
          st.acc[4 * half + i] = mfma16_f32(x, p, st.acc[4 * half + i]);
        }
      } else {
        if constexpr (F::kCodes) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float sc, lo;
            pair_of<DT>(vp[gh], e, sc, lo);
            st.off[half] = fmaf(p[e], lo, st.off[half]);
            p[e] *= sc * (1.f / F::kTimes);
            if constexpr (!F::kPlain) st.off[half] = fmaf(p[e], -F::kBias, st.off[half]);
          }
        }
        bf16x8 b[F::NTV];
        split_terms<F::NTV>(p, b);
#pragma unroll
        for (int x = 0; x < CL; ++x) {
          bf16x8 bx[F::NTV];
          asm("" : "+v"(mine[x]));   // (one register for the mask, not one for each word)
#pragma unroll
          for (int n = 0; n < F::NTV; ++n) {
            u32x4 t = __builtin_bit_cast(u32x4, b[n]);
            if constexpr (CL > 1) {
#pragma unroll
              for (int i = 0; i < 4; ++i) t[i] &= mine[x];
            }
            bx[n] = __builtin_bit_cast(bf16x8, t);
          }
#pragma unroll
          for (int i0 = 0; i0 < 4; i0 += kInTurn) {
            bf16x8 a[kInTurn];
#pragma unroll
            for (int i = 0; i < kInTurn; ++i) a[i] = operand<DT, BITS>(vc[x][gh], i0 + i, cst);
#pragma unroll
            for (int n = 0; n < F::NTV; ++n)
#pragma unroll
              for (int i = 0; i < kInTurn; ++i) st.acc[4 * half + i0 + i] = mfma16(a[i], bx[n], st.acc[4 * half + i0 + i]);
          }
        }
      }
    }
  }
};

// A tile of the tail: rows of 128 elements one after another, `rows` of them in use.  All of it is asked for at once, through
// resources that end with the last row in use: what lies behind it may be anything, and is zeros here (the logits are masked).
// (Whole offsets are the lanes': a scalar part takes no part in the comparison with a resource's end.)
// The columns of the first class attend to it; `mine`: this lane's is one of them.
template <int DT>
__device__ __forceinline__ void tail_tile(const char *kt, const char *vt, int rows, bool mine, int m, int h, const char *q_lds,
                                          float scale, State &st) {
  using E = Elem<DT>;
  constexpr int EB = E::EB, RB = kD * EB, W = EB / 2;   // W: 16-byte pieces of eight channels
  const auto kr = __builtin_amdgcn_make_buffer_rsrc((void *)kt, (short)0, rows * RB, 0x00027000);
  const auto vr = __builtin_amdgcn_make_buffer_rsrc((void *)vt, (short)0, rows * RB, 0x00027000);
  u32x4 kx[4][4][W];
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int w = 0; w < W; ++w)
        kx[s][j][w] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kr, m * RB + 8 * h * EB + (s * 32 * EB + w * 16 + 16 * j * RB), 0, 0));
  uint32_t vx[4][8][2 * W];   // four channels of each of the lane's eight rows, per half of the rows and of the channels
#pragma unroll
  for (int gh = 0; gh < 4; ++gh)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = 4 * h * RB + 4 * m * EB + ((gh & 1) * 64 * EB + (32 * (gh >> 1) + 16 * (e >> 2) + (e & 3)) * RB);
      if constexpr (DT == THK_F32) {
        const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, at, 0, 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) vx[gh][e][i] = x[i];
      } else {
        const uint64_t x = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(vr, at, 0, 0));
        vx[gh][e][0] = (uint32_t)x;
        vx[gh][e][1] = (uint32_t)(x >> 32);
      }
    }
  f32x4 z[4] = {};
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = E::load1(q_lds, 32 * s + 8 * h + e);
    bf16x8 b[1];
    if constexpr (DT == THK_BF16) split_terms<1>(q, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == THK_F32) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(kx[s][j][e >> 2][e & 3]);
        z[j] = mfma16_f32(x, q, z[j]);
      } else {
        z[j] = mfma16(__builtin_bit_cast(bf16x8, kx[s][j][0]), b[0], z[j]);
      }
    }
  }
  softmax_step(z, mine ? rows : 0, h, scale, st);
#pragma unroll
  for (int gh = 0; gh < 4; ++gh) {
    const int g = gh >> 1, half = gh & 1;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = z[2 * g + (e >> 2)][e & 3];
    if constexpr (DT == THK_F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(vx[gh][e][i]);
        st.acc[4 * half + i] = mfma16_f32(x, p, st.acc[4 * half + i]);
      }
    } else {
      bf16x8 b[2];
      split_terms<2>(p, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 x;
#pragma unroll
        for (int w = 0; w < 4; ++w)   // the lower or the upper halves of two rows' words
          x[w] = __builtin_amdgcn_perm(vx[gh][2 * w + 1][i >> 1], vx[gh][2 * w][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int n = 0; n < 2; ++n) st.acc[4 * half + i] = mfma16(__builtin_bit_cast(bf16x8, x), b[n], st.acc[4 * half + i]);
      }
    }
  }
}

constexpr int kRec = kD + 2;     // floats of a split record: max, sum, acc[128]
constexpr int kAccPitch = kD + 4;

// As many zeros as a tile of codes has bytes at most (128 channels, 8 bits, fp32 parameters).
static __device__ __align__(16) const char no_parameters[paged_layout(THK_F32, 8, kD).tile_bytes] = {};


// The lane's number, asked for anew.
__device__ __forceinline__ int lane_again() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

// Inclusive sums over the wave's lanes.
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);   // 1, 2, 4, 8 lanes up within a row of 16
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);   // the row below's last lane
  x += __builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);   // the lower half's last lane
  return x;
}

// How the sequences are cut into pieces: a sequence of t tiles (at least one: an empty one has an output too) into
// ceil(t / per) of them.  Blocks are numbered by sequence, unit and group, piece.
// With per given, every unit has n_split blocks, and those past its last piece have nothing to do.  A block knows its place
// without the lengths.
// Otherwise the cutting is done here, where the lengths are: per = all sequences' tiles over (sequences * n_split), or so much
// more that sequences of different lengths have n_split pieces on average after rounding (300 ragged batches: 9 % longer without
// that, some compute units having a block more); pieces of one sequence of equal size up to a tile; never more than n_split + 1
// per unit and group on average.  The block's place takes a trip to memory and some 100 to 200 instructions (0.8 us), but the
// pieces do not depend on how far the host's bound of the lengths is from the lengths, and one long sequence among short ones is
// cut into as many as it takes.  That is so where the host plans for two pieces or more (paged_by_lengths): a sequence is not cut
// in calls of so many units that it plans for one.
struct Cutting {
  const PagedDecodeArgs &a;
  uint32_t per;   // tiles

  __device__ __forceinline__ uint32_t tiles_of(int rows) const {
    return (uint32_t)max((min(max(rows, 0), (int)a.S) + (kTile - 1)) / kTile, 1);   // S < 2^31 - 63
  }
  // of sequence b; 0 past the last
  __device__ __forceinline__ uint32_t tiles_at(int b) const { return b < a.p.B ? tiles_of(a.s_pages[b]) : 0u; }
  __device__ __forceinline__ uint32_t pieces_of(uint32_t tiles) const { return (tiles + per - 1) / per; }

  __device__ __forceinline__ Cutting(const PagedDecodeArgs &args, int lane) : a(args), per((uint32_t)args.per) {
    if (a.per != 0) return;
    const double want = (double)a.p.B * (double)a.n_split;
    double total = 0;   // exact
    for (int b0 = 0; b0 < a.p.B; b0 += kWave) total += (double)(uint32_t)__builtin_amdgcn_readlane((int)wave_sums(tiles_at(b0 + lane)), 63);
    per = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)ceil(total / want));
    // Sequences of different lengths now have up to a piece more each than they should; longer pieces, until the sum is met.
    for (int i = 0; i < 4; ++i) {
      double have = 0;
      for (int b0 = 0; b0 < a.p.B; b0 += kWave)
        have += (double)(uint32_t)__builtin_amdgcn_readlane((int)wave_sums(pieces_of(tiles_at(b0 + lane))), 63);
      if (have <= want) return;
      per = max(per + 1, (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(per * have / want)));
    }
  }
  // The sequence in which the x-th of all sequences' pieces lies (b = B: none), and the number of pieces in front of it; or,
  // with x < 0, the number of pieces in front of sequence b.  (Not with per given.)
  __device__ __forceinline__ void find(int x, int &b, uint32_t &before, int lane) const {
    before = 0;
    for (int b0 = 0; b0 < a.p.B; b0 += kWave) {
      const uint32_t n = pieces_of(tiles_at(b0 + lane)), sums = wave_sums(n);
      // (lanes past the last sequence have no tiles and no pieces)
      const unsigned long long past = x >= 0 ? __ballot(before + sums > (uint32_t)x) : (b < b0 + kWave ? ~0ull << (b - b0) : 0ull);
      if (past != 0) {
        const int i = __builtin_ctzll(past);
        b = b0 + i;
        before += (uint32_t)__builtin_amdgcn_readlane((int)(sums - n), i);
        return;
      }
      before += (uint32_t)__builtin_amdgcn_readlane((int)sums, 63);
    }
    b = a.p.B;
  }
};

// One block: up to 16 query heads of one unit, one piece of the sequence's tiles, which its four waves take in turn, `step`
// tiles at a time.  The sequence's last piece takes the tail as well.
// Short calls are a chain of trips to memory; everything that depends on the arguments alone is asked for first: the
// lengths, the page of the wave's first tiles, the query, the index list.
template <int DT, int BITS, int NST, int CL>
__global__ __launch_bounds__(256, DT == THK_F32 ? 1 : 2) void k_paged_decode(PagedDecodeArgs a) {
  using E = Elem<DT>;
  using F = Format<DT, BITS>;
  constexpr int EB = E::EB, QP = kD * EB + 16, HC = 16 / CL;   // HC: heads of a class
  constexpr int QN = HC * (kD * EB / 16) / 256 > 0 ? HC * (kD * EB / 16) / 256 : 1;   // 16-byte pieces of the query per thread
  __shared__ __align__(16) char q_lds[HC * QP];
  __shared__ __align__(16) int16_t idx_lds[kD];
  __shared__ __align__(16) float acc_lds[4][16][kAccPitch];
  __shared__ f32x2 ml_lds[4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, h = lane >> 4;
  const int cls = m / HC, hd = m % HC;
  // (a grid has fewer than 2^24 blocks)
  const Cutting cut(a, lane);
  int b;
  uint32_t col, sp, share, n;   // n: pieces of the unit, once its length is known
  if (a.per != 0) {
    const uint32_t x = a.by_split.of(blockIdx.x);
    sp = blockIdx.x - x * (uint32_t)a.n_split;
    b = (int)a.by_cols.of(x);
    col = x - (uint32_t)b * (uint32_t)a.cols;
    share = (uint32_t)a.per;
    n = 0;
  } else {
    uint32_t before;
    cut.find((int)a.by_cols.of(blockIdx.x), b, before, lane);
    if (b >= a.p.B) return;   // more blocks than pieces
    const uint32_t all = cut.tiles_of(scalar_load(a.s_pages, b)), at = blockIdx.x - before * (uint32_t)a.cols;
    n = cut.pieces_of(all);
    col = at / n;
    sp = at - col * n;
    share = (all + n - 1) / n;
  }
  const int s_pages = scalar_load(a.s_pages, b), s_tail = a.s_tail != nullptr ? scalar_load(a.s_tail, b) : 0;
  const uint32_t lh = a.by_groups.of(col), hg = col - lh * (uint32_t)a.groups;
  const uint32_t l = a.p.by_N_kv.of(lh), hk = lh - l * (uint32_t)a.p.N_kv;
  const uint32_t u = (l * (uint32_t)a.p.B + (uint32_t)b) * (uint32_t)a.p.N_kv + hk;
  const UnitPages pages = a.p.unit({l, b, (int)hk});
  // the wave's tiles: t0 + wave * step + x, x < step, then 4 * step on
  const int t0 = (int)min(sp * (uint64_t)share, (uint64_t)(INT32_MAX / kTile));   // (past the sequence's end: none)
  int it = t0 + wave * a.step;
  int page[CL];   // the next tiles' table entries
#pragma unroll
  for (int x = 0; x < CL; ++x) page[x] = pages.page_of(it + x);
  const int heads = min(16, a.G - 16 * (int)hg);
  const int64_t head0 = (int64_t)u * a.G + 16 * hg;   // of all query heads of the call: a unit's are neighbours
  u32x4 qr[QN];   // (heads that are not there: the last one again, zeros later)
#pragma unroll
  for (int i = 0; i < QN; ++i) {
    const int n = (tid + 256 * i) / (kD * EB / 16), c = (tid + 256 * i) % (kD * EB / 16);
    qr[i] = *(const u32x4 *)((const char *)a.q + (head0 + min(n, heads - 1)) * kD * EB + c * 16);
  }
  const int channel = a.idx[(size_t)u * a.T + min(tid, a.T - 1)];

  // (a place without a tile has another one's address; where there is none at all, nothing is read but parameters, and these
  // from the zeros: they meet weights of zero, which must not meet what else memory holds)
  struct Where { const char *t[CL]; GlobalPtr own; int rows, bytes; };
  auto where = [&](int it, int end, int np) {
    Where w;
    const char *any = nullptr;
#pragma unroll
    for (int x = 0; x < CL; ++x) {
      w.t[x] = x < a.step && it + x < end ? pages.in_page(page[x], it + x) : nullptr;
      if (w.t[x] != nullptr) any = w.t[x];
    }
    w.bytes = any != nullptr ? pages.tile_bytes : 0;
    if (any == nullptr) any = no_parameters;
    w.rows = 0;
    w.own = as_global(any) + (uint32_t)(h * (8 * 2 * EB));
#pragma unroll
    for (int x = 0; x < CL; ++x) {
      if (cls == x && w.t[x] != nullptr) {
        w.rows = np - (it + x) * kTile;
        w.own = as_global(w.t[x]) + (uint32_t)(h * (8 * 2 * EB));   // the lane's first group of parameters, less where they begin
      }
      if (w.t[x] == nullptr) w.t[x] = any;
    }
    return w;
  };
  const int np = min(max(s_pages, 0), (int)a.S), nt = min(max(s_tail, 0), a.cap);
  const int t1 = min((np + kTile - 1) / kTile, t0 + (int)share);
  if (n == 0) n = cut.pieces_of(cut.tiles_of(s_pages));
  if (sp >= n) return;
  const bool joined = n > 1, with_tail = sp + 1 == n;   // the last piece takes the tail

  auto ask_pages = [&](int t) {
#pragma unroll
    for (int x = 0; x < CL; ++x) page[x] = pages.page_of(t + x);
  };
  Where cur = where(it, t1, np);
  ask_pages(it + 4 * a.step);
  Tiles<DT, BITS, NST, CL> tl;
  tl.load_keys(cur.t, cur.bytes, cur.own, a.p.lay, m, h);
  tl.template load_values<0, 1>(cur.t, cur.bytes, cur.own, a.p.lay, m, h);
#pragma unroll
  for (int i = 0; i < QN; ++i) {
    const int n = (tid + 256 * i) / (kD * EB / 16), c = (tid + 256 * i) % (kD * EB / 16);
    if (n < HC) *(u32x4 *)(q_lds + n * QP + c * 16) = n < heads ? qr[i] : u32x4{0, 0, 0, 0};
  }
  // kept channels past the last one are the row's padding, which holds zeros
  if (tid < kD) idx_lds[tid] = (int16_t)(tid < a.T ? channel & (kD - 1) : kD);
  if (tid < HC) *(u32x4 *)(q_lds + tid * QP + kD * EB) = u32x4{0, 0, 0, 0};
  __syncthreads();
  const char *const q_row = q_lds + hd * QP;
  Query<DT> q[NST];
#pragma unroll
  for (int s = 0; s < NST; ++s) {
    int16_t c[8];
    *(u32x4 *)c = *(const u32x4 *)(idx_lds + 32 * s + 8 * h);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[s].set(e, E::load1(q_row, c[e]));
  }
  const Mantissa cst;
  State st;
#pragma unroll
  for (int i = 0; i < 8; ++i) st.acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  st.off[0] = st.off[1] = st.l = 0.f;
  st.m = -INFINITY;
  for (; it < t1; it += 4 * a.step) {
    const Where next = where(it + 4 * a.step, t1, np);
    ask_pages(it + 8 * a.step);
    f32x4 z[4];
#pragma unroll
    for (int s = 0; s < NST; ++s) q[s].keep();
    tl.logits(q, cls, cst, z);
    tl.template load_values<1, 2>(cur.t, cur.bytes, cur.own, a.p.lay, m, h);
    softmax_step(z, cur.rows, h, a.scale_log2, st);
    if (!F::kCodes && cur.rows < kTile) tl.template drop_values<0>(cur.rows, h);
    tl.template add_values<0>(z, cls, cst, st);
    tl.load_keys(next.t, next.bytes, next.own, a.p.lay, m, h);
    if (!F::kCodes && cur.rows < kTile) tl.template drop_values<1>(cur.rows, h);
    tl.template add_values<1>(z, cls, cst, st);
    tl.template load_values<0, 1>(next.t, next.bytes, next.own, a.p.lay, m, h);
    cur = next;
  }
  // The arguments that are needed from here on are asked for here: kept through the loop they cost it registers.
  typedef const __attribute__((address_space(4))) PagedDecodeArgs LateArgs;
  LateArgs *late = (LateArgs *)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(late));
  LateArgs &z = *late;
  const int heads2 = min(16, z.G - 16 * (int)hg);
  const int64_t head2 = (int64_t)u * z.G + 16 * hg;
  if (with_tail)
    for (int r0 = (3 - wave) * kTile; r0 < nt; r0 += 4 * kTile) {   // (the last wave has the fewest pages)
      const size_t at = ((size_t)u * z.cap + r0) * kD * EB;
      tail_tile<DT>((const char *)z.kt + at, (const char *)z.vt + at, min(kTile, nt - r0), cls == 0, m, h, q_row, z.scale_log2, st);
    }
  st.l = sum_quarters(st.l);
  if constexpr (F::kCodes) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float off = sum_quarters(st.off[half]);
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[4 * half + i] += off;
    }
  }
  const int lane2 = lane_again(), m2 = lane2 & 15, h2 = lane2 >> 4;   // (not kept through the loops: registers)
  if (m2 % HC < heads2) {
    if (h2 == 0) ml_lds[wave][m2] = f32x2{st.m, st.l};
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(f32x4 *)&acc_lds[wave][m2][64 * half + 16 * h2 + 4 * r] =
            f32x4{st.acc[4 * half][r], st.acc[4 * half + 1][r], st.acc[4 * half + 2][r], st.acc[4 * half + 3][r]};
  }
  __syncthreads();
  // the states of a head, joined by a wave, two channels a lane: four waves, CL columns of each
  for (int n = wave; n < heads2; n += 4) {
    f32x2 ml[4][CL], x[4][CL];
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int c = 0; c < CL; ++c) {
        ml[w][c] = ml_lds[w][c * HC + n];
        x[w][c] = *(const f32x2 *)&acc_lds[w][c * HC + n][2 * lane2];
        M = fmaxf(M, ml[w][c][0]);
      }
    f32x2 o = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int c = 0; c < CL; ++c) {
        const float wgt = ml[w][c][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w][c][0] - M);
        L = fmaf(ml[w][c][1], wgt, L);
        o += x[w][c] * wgt;
      }
    if (!joined) {
      const float inv = L > 0.f ? 1.f / L : 0.f;   // no rows at all: zeros
      E::store2((void *)as_global(z.out), (head2 + n) * kD + 2 * lane2, o[0] * inv, o[1] * inv);
    } else {
      float *const rec = (float *)as_global(z.ws) + ((int64_t)blockIdx.x * min(z.G, 16) + n) * kRec;
      *(f32x2 *)(rec + 2 + 2 * lane2) = o;
      if (lane2 == 0) *(f32x2 *)rec = f32x2{M, L};
    }
  }
}

// The pieces of one query head, joined: a block per head, its NW waves take eight records at a time, a lane two channels:
//   M = max M_i,  out = sum 2^(M_i - M) acc_i / sum 2^(M_i - M) l_i.
// One wave for up to 8 pieces, four up to 32, eight beyond: all records are on their way at once.  Its time is its launch and two
// trips to memory (2.1 to 3 us after a short call, 4 to 5 where the cutting is done again).  Joined inside the first launch, by
// the last block of a head to arrive, calls were 0.3 to 1 us slower: the arrival is a trip of its own.
template <int DT, int NW>
__global__ __launch_bounds__(64 * NW) void k_paged_merge(PagedDecodeArgs a) {
  constexpr int P = 8;
  __shared__ f32x2 part[NW][kWave], part_ml[NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t head = blockIdx.x, u = head / (uint32_t)a.G, n = head - u * (uint32_t)a.G;
  const UnitPlace place = a.p.place(u);
  int b = place.b;
  const Cutting cut(a, lane);
  const int pieces = (int)cut.pieces_of(cut.tiles_of(scalar_load(a.s_pages, b)));
  if (pieces == 1) return;   // written by the piece itself
  uint32_t before = (uint32_t)(b * a.n_split), blocks = (uint32_t)a.n_split;   // blocks of a unit and group
  if (a.per == 0) {
    cut.find(-1, b, before, lane);
    blocks = (uint32_t)pieces;
  }
  const uint32_t col = (place.l * (uint32_t)a.p.N_kv + (uint32_t)place.h) * (uint32_t)a.groups + n / 16;
  const int64_t stride = (int64_t)min(a.G, 16) * kRec;   // from piece to piece
  const float *const rec = a.ws + (int64_t)(before * (uint32_t)a.cols + col * blocks) * stride + (n & 15) * kRec;
  float M = -INFINITY, L = 0.f;
  f32x2 o = {0.f, 0.f};
  for (int i0 = wave * P; i0 < pieces; i0 += NW * P) {
    f32x2 ml[P], x[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {   // (records past the last: the last one again, without weight)
      const float *const r = rec + min(i0 + i, pieces - 1) * stride;
      ml[i] = *(const f32x2 *)r;
      x[i] = *(const f32x2 *)(r + 2 + 2 * lane);
    }
    float M_new = M;
#pragma unroll
    for (int i = 0; i < P; ++i) M_new = fmaxf(M_new, ml[i][0]);
    const float keep = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - M_new);
    M = M_new;
    L *= keep;
    o *= keep;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float wgt = i0 + i >= pieces || ml[i][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i][0] - M);
      L = fmaf(ml[i][1], wgt, L);
      o += x[i] * wgt;
    }
  }
  part[wave][lane] = o;
  if (lane == 0) part_ml[wave] = f32x2{M, L};
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, part_ml[w][0]);
  L = 0.f;
  o = f32x2{0.f, 0.f};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const f32x2 ml = part_ml[w];
    const float wgt = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - M);
    L = fmaf(ml[1], wgt, L);
    o += part[w][lane] * wgt;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  Elem<DT>::store2(a.out, (int64_t)head * kD + 2 * lane, o[0] * inv, o[1] * inv);
}

// CL: tiles a wave takes at once, as paged_decode_step allows them for T channels.
template <int DT, int BITS, int CL, int MOST_STEPS>
void (*kernel_of(int T))(PagedDecodeArgs) {
  if constexpr (MOST_STEPS == 4)
    if (T > 96) return k_paged_decode<DT, BITS, 4, CL>;
  return T <= 64 ? k_paged_decode<DT, BITS, 2, CL> : k_paged_decode<DT, BITS, 3, CL>;
}

template <int DT, int BITS>
hipError_t launch(const PagedDecodeArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  void (*k)(PagedDecodeArgs) = nullptr;
  const int CL = a.step > 2 ? 4 : a.step;   // (tiles past a.step are columns without weight: no more of them than needed)
  if (CL == 1) k = kernel_of<DT, BITS, 1, 4>(a.T);
  if constexpr (BITS == 4) {
    if (CL == 2) k = kernel_of<DT, BITS, 2, 4>(a.T);
    if (CL == 4) k = kernel_of<DT, BITS, 4, 3>(a.T);
  }
  if constexpr (BITS == 8)
    if (CL == 2) k = kernel_of<DT, BITS, 2, 3>(a.T);
  PagedDecodeArgs copy = a;
  void *args[] = {&copy};
  hipError_t e = launch_main_kernel((const void *)k, dim3((unsigned)(a.units * a.groups * (a.per == 0 ? a.n_split + 1 : a.n_split))), dim3(256), args, 0, st);
  if (e != hipSuccess || a.n_split == 1) return e;
  const dim3 heads((unsigned)(a.units * a.G));
  if (a.n_split <= 8) hipLaunchKernelGGL((k_paged_merge<DT, 1>), heads, dim3(64), 0, st, a);
  else if (a.n_split <= 32) hipLaunchKernelGGL((k_paged_merge<DT, 4>), heads, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_paged_merge<DT, 8>), heads, dim3(512), 0, st, a);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace thk
