// Attention of one new token over a paged cache and a tail: the kernel, for both element types and all page formats.
//
//   z_r = scale * sum_t q_t k_rt,  out = sum_r p_r v_r / sum_r p_r,  p_r = 2^(z_r - m)
// With codes, k_rt = m_t + s_t c_rt (a group's scale and minimum, t a channel of the tile), so
//   z_r = scale * ( sum_t q_t m_t  +  sum_t (q_t s_t) c_rt ):
// the query takes the scales, once per tile, and the codes enter the matrix cores as the whole numbers they are, which
// bf16 holds exactly.  Values likewise: sum_r p_r v_rc = sum_r p_r m_r + sum_r (p_r s_r) c_rc.  What is not exact in bf16 --
// the scaled query and the scaled probabilities -- enters as a sum of bf16 terms: two for bf16 tensors (2^-17 of the value),
// three for fp32 ones (2^-25).  Of a code c an operand holds something more, which is taken out again with the minimum: 4-bit
// codes of bf16 tensors are used as 16 + c, whose bits are the code in the mantissa of 16 (one shift and one mask for two of
// them); all others as c less half the range, a signed byte, which keeps the two sums that make up a logit small and with them
// what their rounding costs (fp32, 8 bits, 2048 rows: 1.5e-6 of the result with plain codes).
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
#pragma once
#include "thk_paged.h"

namespace thk {
namespace paged {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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
  static constexpr float kTimes = BITS == 4 && !kMantissa ? 16.f : 1.f;
  static constexpr float kBias = kMantissa ? 16.f : -128.f;
};

// Signed bytes A and B of x as two bf16 numbers: whole numbers below 256 in size have all their bits in a float's upper half.
template <int A, int B>
__device__ __forceinline__ uint32_t byte_pair(uint32_t x) {
  return __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(x >> (8 * B))), __float_as_uint((float)(int8_t)(x >> (8 * A))), 0x07060302u);
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
__device__ __forceinline__ void load_pairs(const char *par, u32x4 (&w)[DT == THK_BF16 ? 2 : 4]) {
#pragma unroll
  for (int i = 0; i < (DT == THK_BF16 ? 2 : 4); ++i) w[i] = ((const u32x4 *)par)[i];
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
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (16 * j + 4 * h + i >= rows) z[j][i] = -INFINITY;
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
};
template <>
struct Query<THK_BF16> {
  bf16x8 x;
  __device__ __forceinline__ float operator[](int e) const { return (float)x[e]; }
  __device__ __forceinline__ void set(int e, float v) { x[e] = (__bf16)v; }   // exact: v is an element
};

// CL tiles of pages: t[x] is the x-th (any tile again where there is none).  `rows`: rows that count in the lane's own tile,
// `own`: that tile's first byte, cls: its place x.
template <int DT, int BITS, int NST, int CL>
__device__ __forceinline__ void page_tiles(const char *const (&t)[CL], const char *own, int cls, int rows, const PagedLayout &lay,
                                           int m, int h, const Query<DT> (&q)[NST], float scale, const Mantissa &cst, State &st) {
  using F = Format<DT, BITS>;
  constexpr int NP = DT == THK_BF16 ? 2 : 4;
  u32x4 kc[CL][NST][F::NC], kp[F::kCodes ? NST : 1][NP];
#pragma unroll
  for (int s = 0; s < NST; ++s) {
    const int c = min(4 * s + h, lay.chunks - 1);   // groups past the last meet zeros of the query
    if constexpr (F::kCodes) load_pairs<DT>(own + (uint32_t)(lay.k_params + c * 8 * 2 * Elem<DT>::EB), kp[s]);
    const uint32_t at = (uint32_t)(c * 64 * F::UB + m * 16);   // 32 bits behind a scalar base
#pragma unroll
    for (int x = 0; x < CL; ++x)
#pragma unroll
      for (int k = 0; k < F::NC; ++k) kc[x][s][k] = ld_stream((const u32x4 *)(t[x] + at + k * 256));
  }
  // with codes all of the values are asked for here as well
  // (the parameters after the first product where the registers would not hold them: 128 channels, two tiles)
  constexpr bool kLate = NST == 4 && CL == 2;
  u32x4 vc[F::kCodes ? CL : 1][F::kCodes ? 4 : 1][F::NC], vp[F::kCodes ? 4 : 1][NP];
  const uint32_t pat = (uint32_t)(lay.v_params + h * 2 * 8 * 2 * Elem<DT>::EB);
  auto load_value_pairs = [&] {
#pragma unroll
    for (int gh = 0; gh < 4; ++gh) load_pairs<DT>(own + pat + ((gh >> 1) * 8 + (gh & 1)) * 8 * 2 * Elem<DT>::EB, vp[gh]);
  };
  if constexpr (F::kCodes) {
    if constexpr (!kLate) load_value_pairs();
    const uint32_t at = (uint32_t)(lay.v_codes + h * 2 * 64 * F::UB + m * 16);
#pragma unroll
    for (int gh = 0; gh < 4; ++gh) {
      const int grp = (gh >> 1) * 8 + (gh & 1);   // the lane's group, less 2 h
#pragma unroll
      for (int x = 0; x < CL; ++x)
#pragma unroll
        for (int k = 0; k < F::NC; ++k) vc[x][gh][k] = ld_stream((const u32x4 *)(t[x] + at + grp * 64 * F::UB + k * 256));
    }
  }
  // the operands are made where they are used, not ahead: they would not fit into the registers
  __builtin_amdgcn_sched_barrier(0);
  f32x4 zx[CL][4] = {};
  float off = 0.f;
#pragma unroll
  for (int s = 0; s < NST; ++s) {
    if constexpr (F::kFp32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(kc[0][s][2 * j + (e >> 2)][e & 3]);
        zx[0][j] = mfma16_f32(x, q[s].x, zx[0][j]);
      }
    } else {
      bf16x8 b[F::NTK];
      if constexpr (F::kCodes) {
        float qs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float sc, lo;
          pair_of<DT>(kp[s], e, sc, lo);
          off = fmaf(q[s][e], lo, off);
          qs[e] = q[s][e] * (sc * (1.f / F::kTimes));
          off = fmaf(qs[e], -F::kBias, off);
        }
        split_terms<F::NTK>(qs, b);
      } else {
        b[0] = q[s].x;
      }
#pragma unroll
      for (int x = 0; x < CL; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 a = operand<DT, BITS>(kc[x][s], j, cst);
#pragma unroll
          for (int n = 0; n < F::NTK; ++n) zx[x][j] = mfma16(a, b[n], zx[x][j]);
        }
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (F::kCodes && kLate) load_value_pairs();
  f32x4 z[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    z[j] = zx[0][j];
#pragma unroll
    for (int x = 1; x < CL; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) z[j][i] = cls == x ? zx[x][j][i] : z[j][i];
  }
  if constexpr (F::kCodes) {
    off = sum_quarters(off);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] += off;
  }
  softmax_step(z, rows, h, scale, st);
#pragma unroll
  for (int gh = 0; gh < 4; ++gh) {
    const int g = gh >> 1, half = gh & 1;
    if constexpr (F::kCodes) __builtin_amdgcn_sched_barrier(0);
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = z[2 * g + (e >> 2)][e & 3];
    if constexpr (F::kCodes) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float sc, lo;
        pair_of<DT>(vp[gh], e, sc, lo);
        st.off[half] = fmaf(p[e], lo, st.off[half]);
        p[e] *= sc * (1.f / F::kTimes);
        st.off[half] = fmaf(p[e], -F::kBias, st.off[half]);
      }
      bf16x8 b[F::NTV];
      split_terms<F::NTV>(p, b);
#pragma unroll
      for (int x = 0; x < CL; ++x) {
        bf16x8 bx[F::NTV];
#pragma unroll
        for (int n = 0; n < F::NTV; ++n) {
          u32x4 w = __builtin_bit_cast(u32x4, b[n]);
          if constexpr (CL > 1) w &= cls == x ? 0xffffffffu : 0u;
          bx[n] = __builtin_bit_cast(bf16x8, w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bf16x8 a = operand<DT, BITS>(vc[x][gh], i, cst);
#pragma unroll
          for (int n = 0; n < F::NTV; ++n) st.acc[4 * half + i] = mfma16(a, bx[n], st.acc[4 * half + i]);
        }
      }
    } else {
      u32x4 vw[F::NC];
#pragma unroll
      for (int k = 0; k < F::NC; ++k)
        vw[k] = ld_stream((const u32x4 *)(t[0] + (uint32_t)(lay.v_codes + ((g * 4 + h) * 2 + half) * 64 * F::UB + m * 16) + k * 256));
      if constexpr (F::kFp32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(vw[2 * i + (e >> 2)][e & 3]);
          st.acc[4 * half + i] = mfma16_f32(x, p, st.acc[4 * half + i]);
        }
      } else {
        bf16x8 b[F::NTV];
        split_terms<F::NTV>(p, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bf16x8 a = operand<DT, BITS>(vw, i, cst);
#pragma unroll
          for (int n = 0; n < F::NTV; ++n) st.acc[4 * half + i] = mfma16(a, b[n], st.acc[4 * half + i]);
        }
      }
    }
  }
}

// A tile of the tail: rows of 128 elements one after another, `rows` of them in use.  Rows past that are not read, since
// what lies there may be anything: the last row in use stands in for their keys (their logits are masked) and zeros for
// their values.  The columns of the first class attend to it; `mine`: this lane's is one of them.
template <int DT>
__device__ __forceinline__ void tail_tile(const char *kt, const char *vt, int rows, bool mine, int m, int h, const char *q_lds,
                                          float scale, State &st) {
  using E = Elem<DT>;
  constexpr int EB = E::EB;
  f32x4 z[4] = {};
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = E::load1(q_lds, 32 * s + 8 * h + e);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const char *const row = kt + (size_t)min(16 * j + m, rows - 1) * kD * EB + (32 * s + 8 * h) * EB;
      if constexpr (DT == THK_F32) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = ((const float *)row)[e];
        z[j] = mfma16_f32(x, q, z[j]);
      } else {
        bf16x8 b[1];
        split_terms<1>(q, b);
        z[j] = mfma16(__builtin_bit_cast(bf16x8, *(const u32x4 *)row), b[0], z[j]);
      }
    }
  }
  softmax_step(z, mine ? rows : 0, h, scale, st);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    if (32 * g >= rows) break;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float p[8];
      uint32_t x[8][DT == THK_F32 ? 4 : 2];   // four channels of each of the lane's eight rows
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = z[2 * g + (e >> 2)][e & 3];
        const int r = 32 * g + 16 * (e >> 2) + 4 * h + (e & 3);
        const char *const row = vt + (size_t)min(r, rows - 1) * kD * EB + (64 * half + 4 * m) * EB;
#pragma unroll
        for (int i = 0; i < (DT == THK_F32 ? 4 : 2); ++i) x[e][i] = r < rows ? ((const uint32_t *)row)[i] : 0u;
      }
      if constexpr (DT == THK_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float a[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = __uint_as_float(x[e][i]);
          st.acc[4 * half + i] = mfma16_f32(a, p, st.acc[4 * half + i]);
        }
      } else {
        bf16x8 b[2];
        split_terms<2>(p, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4 a;
#pragma unroll
          for (int w = 0; w < 4; ++w)   // the lower or the upper halves of two rows' words
            a[w] = __builtin_amdgcn_perm(x[2 * w + 1][i >> 1], x[2 * w][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int n = 0; n < 2; ++n) st.acc[4 * half + i] = mfma16(__builtin_bit_cast(bf16x8, a), b[n], st.acc[4 * half + i]);
        }
      }
    }
  }
}

constexpr int kRec = kD + 2;     // floats of a split record: max, sum, acc[128]
constexpr int kAccPitch = kD + 4;

// One block: up to 16 query heads of one unit, one piece of the sequence's tiles, shared out among its four waves.  The
// sequence's last piece takes the tail as well.
template <int DT, int BITS, int NST, int CL>
__global__ __launch_bounds__(256, DT == THK_F32 && BITS != 0 ? 1 : 2) void k_paged_decode(PagedDecodeArgs a) {
  using E = Elem<DT>;
  constexpr int EB = E::EB, QP = kD * EB + 16, HC = 16 / CL;   // HC: heads of a class
  __shared__ __align__(16) union {
    struct { char q[HC * QP]; int16_t idx[kD]; } in;
    struct { float acc[4][16][kAccPitch], ml[4][16][2]; } out;
  } lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, h = lane >> 4;
  const int cls = m / HC, hd = m % HC;
  const int sp = blockIdx.x % (uint32_t)a.n_split;
  const int64_t ug = blockIdx.x / (uint32_t)a.n_split;
  const int hg = (int)(ug % a.groups);
  const int64_t u = ug / a.groups;
  const int hk = (int)(u % a.p.N_kv), b = (int)(u / a.p.N_kv % a.p.B);
  const int64_t l = u / a.p.N_kv / a.p.B;
  const int heads = min(16, a.G - 16 * hg);
  const int64_t head0 = u * a.G + 16 * hg;   // of all query heads of the call: a unit's are neighbours
  const int np = (int)min((int64_t)max(a.s_pages[b], 0), a.S);
  const int nt = a.s_tail != nullptr ? min(max(a.s_tail[b], 0), a.cap) : 0;
  const int tiles = (np + kTile - 1) / kTile;
  const int last = max(0, (tiles - 1) / a.tiles_per_split);   // the piece that also takes the tail
  if (sp > last) return;
  const int t0 = sp * a.tiles_per_split, t1 = min(tiles, t0 + a.tiles_per_split);

  for (int i = tid; i < HC * (kD * EB / 16); i += 256) {
    const int n = i / (kD * EB / 16), c = i % (kD * EB / 16);
    u32x4 x = {0, 0, 0, 0};
    if (n < heads) x = *(const u32x4 *)((const char *)a.q + (head0 + n) * kD * EB + c * 16);
    *(u32x4 *)(lds.in.q + n * QP + c * 16) = x;
  }
  if (tid < kD) lds.in.idx[tid] = tid < a.T ? a.idx[u * a.T + tid] & (kD - 1) : -1;
  __syncthreads();
  const char *const q_row = lds.in.q + hd * QP;
  Query<DT> q[NST];
#pragma unroll
  for (int s = 0; s < NST; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = lds.in.idx[32 * s + 8 * h + e];
      q[s].set(e, c >= 0 ? E::load1(q_row, c) : 0.f);
    }
  const Mantissa cst;
  State st;
#pragma unroll
  for (int i = 0; i < 8; ++i) st.acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  st.off[0] = st.off[1] = st.l = 0.f;
  st.m = -INFINITY;
  const int each = (t1 - t0 + 3) / 4, w0 = t0 + wave * each, w1 = min(t1, w0 + each);   // this wave's tiles
  for (int it = w0; it < w1; it += CL) {
    const char *t[CL], *any = nullptr;
#pragma unroll
    for (int x = 0; x < CL; ++x) {
      t[x] = it + x < w1 ? a.p.tile(l, b, hk, it + x) : nullptr;
      if (t[x] != nullptr) any = t[x];
    }
    if (any == nullptr) continue;
    int rows = 0;
    const char *own = any;
#pragma unroll
    for (int x = 0; x < CL; ++x) {
      if (cls == x && t[x] != nullptr) {
        rows = np - (it + x) * kTile;
        own = t[x];
      }
      if (t[x] == nullptr) t[x] = any;
    }
    page_tiles<DT, BITS, NST, CL>(t, own, cls, rows, a.p.lay, m, h, q, a.scale_log2, cst, st);
  }
  if (sp == last)
    for (int r0 = wave * kTile; r0 < nt; r0 += 4 * kTile) {
      const size_t at = ((size_t)u * a.cap + r0) * kD * EB;
      tail_tile<DT>((const char *)a.kt + at, (const char *)a.vt + at, min(kTile, nt - r0), cls == 0, m, h, q_row, a.scale_log2, st);
    }
  st.l = sum_quarters(st.l);
  if constexpr (BITS != 0) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float off = sum_quarters(st.off[half]);
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[4 * half + i] += off;
    }
  }
  __syncthreads();   // the query's part of LDS is not needed any more
  if (h == 0) {
    lds.out.ml[wave][m][0] = st.m;
    lds.out.ml[wave][m][1] = st.l;
  }
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *(f32x4 *)&lds.out.acc[wave][m][64 * half + 16 * h + 4 * r] =
          f32x4{st.acc[4 * half][r], st.acc[4 * half + 1][r], st.acc[4 * half + 2][r], st.acc[4 * half + 3][r]};
  __syncthreads();
  // the states of a head, joined: four waves, CL columns of each
  const int n = tid >> 4, c0 = (tid & 15) * 8;
  if (n >= heads) return;
  float M = -INFINITY, L = 0.f, o[8] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int x = 0; x < CL; ++x) M = fmaxf(M, lds.out.ml[w][x * HC + n][0]);
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int x = 0; x < CL; ++x) {
      const int col = x * HC + n;
      const float mw = lds.out.ml[w][col][0], wgt = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M);
      L = fmaf(lds.out.ml[w][col][1], wgt, L);
#pragma unroll
      for (int c = 0; c < 8; ++c) o[c] = fmaf(lds.out.acc[w][col][c0 + c], wgt, o[c]);
    }
  if (last > 0) {
    float *const rec = a.ws + ((head0 + n) * a.n_split + sp) * kRec;
    if (c0 == 0) *(f32x2 *)rec = f32x2{M, L};
#pragma unroll
    for (int c = 0; c < 8; c += 2) *(f32x2 *)(rec + 2 + c0 + c) = f32x2{o[c], o[c + 1]};
    return;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;   // no rows at all: zeros
#pragma unroll
  for (int c = 0; c < 8; c += 2) E::store2(a.out, (head0 + n) * kD + c0 + c, o[c] * inv, o[c + 1] * inv);
}

// The pieces of one query head, joined: a block per head, its four waves take the records in turn, a lane two channels.
template <int DT>
__global__ __launch_bounds__(256) void k_paged_merge(PagedDecodeArgs a) {
  __shared__ f32x2 part[4][kWave], part_ml[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t head = blockIdx.x;
  const int b = (int)(head / a.G / a.p.N_kv % a.p.B);
  const int np = (int)min((int64_t)max(a.s_pages[b], 0), a.S);
  const int pieces = max(0, ((np + kTile - 1) / kTile - 1) / a.tiles_per_split) + 1;
  if (pieces == 1) return;   // written by the piece itself
  const float *const rec = a.ws + head * a.n_split * kRec;
  float M = -INFINITY, L = 0.f;
  f32x2 o = {0.f, 0.f};
  for (int i = wave; i < pieces; i += 4) {
    const f32x2 ml = *(const f32x2 *)(rec + i * kRec), x = *(const f32x2 *)(rec + i * kRec + 2 + 2 * lane);
    const float M_new = fmaxf(M, ml[0]);
    const float keep = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - M_new), wgt = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - M_new);
    M = M_new;
    L = L * keep + ml[1] * wgt;
    o = o * keep + x * wgt;
  }
  part[wave][lane] = o;
  if (lane == 0) part_ml[wave] = f32x2{M, L};
  __syncthreads();
  if (wave != 0) return;
  for (int w = 0; w < 4; ++w) M = fmaxf(M, part_ml[w][0]);
  L = 0.f;
  o = f32x2{0.f, 0.f};
  for (int w = 0; w < 4; ++w) {
    const f32x2 ml = part_ml[w];
    const float wgt = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - M);
    L += ml[1] * wgt;
    o += part[w][lane] * wgt;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  Elem<DT>::store2(a.out, head * kD + 2 * lane, o[0] * inv, o[1] * inv);
}

template <int DT, int BITS, int CL>
void (*kernel_of(int T))(PagedDecodeArgs) {
  return T <= 64 ? k_paged_decode<DT, BITS, 2, CL> : T <= 96 ? k_paged_decode<DT, BITS, 3, CL> : k_paged_decode<DT, BITS, 4, CL>;
}

template <int DT, int BITS>
hipError_t launch(const PagedDecodeArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  void (*k)(PagedDecodeArgs);
  if constexpr (BITS == 4) k = a.G <= 8 ? kernel_of<DT, BITS, 2>(a.T) : kernel_of<DT, BITS, 1>(a.T);
  else k = kernel_of<DT, BITS, 1>(a.T);
  PagedDecodeArgs copy = a;
  void *args[] = {&copy};
  hipError_t e = launch_main_kernel((const void *)k, dim3((unsigned)(a.units * a.groups * a.n_split)), dim3(256), args, 0, st);
  if (e != hipSuccess || a.n_split == 1) return e;
  hipLaunchKernelGGL(k_paged_merge<DT>, dim3((unsigned)(a.units * a.G)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace thk
