// Attention of one new token over a paged cache and a tail: the kernel, for both element types and all page formats.
//
//   z_r = scale * sum_t q_t k_rt,  out = sum_r p_r v_r / sum_r p_r,  p_r = 2^(z_r - m)
// With codes, k_rt = m_t + s_t c_rt (a group's scale and minimum, t a channel of the tile), so
//   z_r = scale * ( sum_t q_t m_t  +  sum_t (q_t s_t) c_rt ):
// the query takes the scales, once per tile, and the codes enter the matrix cores as the whole numbers they are, which
// bf16 holds exactly.  Values likewise: sum_r p_r v_rc = sum_r p_r m_r + sum_r (p_r s_r) c_rc.  What is not exact in bf16 --
// the scaled query and the scaled probabilities -- enters as a sum of bf16 terms: two for bf16 tensors (2^-17 of the value),
// three for fp32 ones (2^-25).  4-bit codes are used as 16 + c, whose bits are the code in the mantissa of 16; the 16 is taken
// out again with the minimum.
//
// A wave takes a tile of 64 rows at a time.  S^T = K q^T: A = 16 rows x 32 channels of keys, B = 32 channels x 16 query
// heads, so lane (m, h) = (lane % 16, lane / 16) ends up with the logits of head m for rows 16 j + 4 h + i.  out^T = V^T P^T:
// B = 32 rows x 16 heads wants from lane (m, h) eight rows of head m, and the groups of the values are made of just the
// rows the lane holds: the probabilities go from one product into the other in the lane's own registers.  Heads past G are
// columns of zeros.
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
  static constexpr float kBias = BITS == 4 ? 16.f : 0.f;      // what an operand holds above its code
};

// Unit j of a lane's cells as an operand of eight.
template <int DT, int BITS>
__device__ __forceinline__ bf16x8 operand(const u32x4 (&w)[Format<DT, BITS>::NC], int j) {
  u32x4 u;
  if constexpr (BITS == 4) {
    const uint32_t x = w[0][j];
    u[0] = ((x << 3) & 0x00780078u) | 0x41804180u;
    u[1] = ((x >> 1) & 0x00780078u) | 0x41804180u;
    u[2] = ((x >> 5) & 0x00780078u) | 0x41804180u;
    u[3] = ((x >> 9) & 0x00780078u) | 0x41804180u;
  } else if constexpr (BITS == 8) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {   // a whole number below 256 as a float has its bits in the upper half
      const uint32_t x = w[j >> 1][2 * (j & 1) + (p >> 1)] >> (16 * (p & 1));
      u[p] = __builtin_amdgcn_perm(__float_as_uint((float)((x >> 8) & 255u)), __float_as_uint((float)(x & 255u)), 0x07060302u);
    }
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

// A wave's running softmax.  acc[4 half + i][r]: channel 64 half + 16 h + 4 r + i of head m.
struct State {
  f32x4 acc[8];
  float off[2];   // this lane's share of sum_r p_r m_r per half of the channels
  float l;        // this lane's share of sum_r p_r
  float m;        // whole number: every change of it scales by an exact power of two
};

// p[j][i] <- 2^(scale z - m) for the tile's logits z, masked past `rows`; the state is brought to the new m.
__device__ __forceinline__ void softmax_step(f32x4 (&z)[4], int rows, int h, float scale, State &st) {
  if (rows < kTile) {
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
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      z[j][i] = __builtin_amdgcn_exp2f(fmaf(z[j][i], scale, -st.m));
      sum += z[j][i];
    }
  st.l += sum;
}

// A tile of pages.  q: this lane's eight channels of head m per step of 32 kept channels (zeros past T).
template <int DT, int BITS, int NST>
__device__ __forceinline__ void page_tile(const char *t, const PagedLayout &lay, int rows, int m, int h,
                                          const float (&q)[NST][8], float scale, State &st) {
  using F = Format<DT, BITS>;
  constexpr int NP = DT == THK_BF16 ? 2 : 4;
  u32x4 kc[NST][F::NC], kp[F::kCodes ? NST : 1][NP];
#pragma unroll
  for (int s = 0; s < NST; ++s) {
    const int c = min(4 * s + h, lay.chunks - 1);   // groups past the last meet zeros of the query
#pragma unroll
    for (int k = 0; k < F::NC; ++k) kc[s][k] = ld_stream((const u32x4 *)(t + c * 64 * F::UB + (k * 16 + m) * 16));
    if constexpr (F::kCodes) load_pairs<DT>(t + lay.k_params + c * 8 * 2 * Elem<DT>::EB, kp[s]);
  }
  f32x4 z[4] = {};
  float off = 0.f;
#pragma unroll
  for (int s = 0; s < NST; ++s) {
    if constexpr (F::kFp32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(kc[s][2 * j + (e >> 2)][e & 3]);
        z[j] = mfma16_f32(x, q[s], z[j]);
      }
    } else {
      float qs[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        qs[e] = q[s][e];
        if constexpr (F::kCodes) {
          float sc, lo;
          pair_of<DT>(kp[s], e, sc, lo);
          off = fmaf(q[s][e], lo, off);
          qs[e] *= sc;
          if constexpr (F::kBias != 0.f) off = fmaf(qs[e], -F::kBias, off);
        }
      }
      bf16x8 b[F::NTK];
      split_terms<F::NTK>(qs, b);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8 a = operand<DT, BITS>(kc[s], j);
#pragma unroll
        for (int n = 0; n < F::NTK; ++n) z[j] = mfma16(a, b[n], z[j]);
      }
    }
  }
  if constexpr (F::kCodes) {
    off = sum_quarters(off);
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] += off;
  }
  softmax_step(z, rows, h, scale, st);
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int grp = (g * 4 + h) * 2 + half;
      u32x4 vc[F::NC];
#pragma unroll
      for (int k = 0; k < F::NC; ++k) vc[k] = ld_stream((const u32x4 *)(t + lay.v_codes + grp * 64 * F::UB + (k * 16 + m) * 16));
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = z[2 * g + (e >> 2)][e & 3];
      if constexpr (F::kFp32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(vc[2 * i + (e >> 2)][e & 3]);
          st.acc[4 * half + i] = mfma16_f32(x, p, st.acc[4 * half + i]);
        }
      } else {
        if constexpr (F::kCodes) {
          u32x4 vp[NP];
          load_pairs<DT>(t + lay.v_params + grp * 8 * 2 * Elem<DT>::EB, vp);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float sc, lo;
            pair_of<DT>(vp, e, sc, lo);
            st.off[half] = fmaf(p[e], lo, st.off[half]);
            p[e] *= sc;
            if constexpr (F::kBias != 0.f) st.off[half] = fmaf(p[e], -F::kBias, st.off[half]);
          }
        }
        bf16x8 b[F::NTV];
        split_terms<F::NTV>(p, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bf16x8 a = operand<DT, BITS>(vc, i);
#pragma unroll
          for (int n = 0; n < F::NTV; ++n) st.acc[4 * half + i] = mfma16(a, b[n], st.acc[4 * half + i]);
        }
      }
    }
}

// A tile of the tail: rows of 128 elements one after another, `rows` of them in use.  Rows past that are not read, since
// what lies there may be anything: the last row in use stands in for their keys (their logits are masked) and zeros for
// their values.
template <int DT>
__device__ __forceinline__ void tail_tile(const char *kt, const char *vt, int rows, int m, int h, const char *q_lds,
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
  softmax_step(z, rows, h, scale, st);
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

// One block: 16 query heads of one unit, one piece of the sequence's tiles; its four waves take the tiles in turn.  The
// sequence's last piece takes the tail as well.
template <int DT, int BITS, int NST>
__global__ __launch_bounds__(256, 2) void k_paged_decode(PagedDecodeArgs a) {
  using E = Elem<DT>;
  constexpr int EB = E::EB, QP = kD * EB + 16;
  __shared__ __align__(16) union {
    struct { char q[16 * QP]; int16_t idx[kD]; } in;
    struct { float acc[4][16][kAccPitch], ml[4][16][2]; } out;
  } lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, h = lane >> 4;
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
  const int items = t1 - t0 + (sp == last ? (nt + kTile - 1) / kTile : 0);

  for (int i = tid; i < 16 * (kD * EB / 16); i += 256) {
    const int n = i / (kD * EB / 16), c = i % (kD * EB / 16);
    u32x4 x = {0, 0, 0, 0};
    if (n < heads) x = *(const u32x4 *)((const char *)a.q + (head0 + n) * kD * EB + c * 16);
    *(u32x4 *)(lds.in.q + n * QP + c * 16) = x;
  }
  if (tid < kD) lds.in.idx[tid] = tid < a.T ? a.idx[u * a.T + tid] & (kD - 1) : -1;
  __syncthreads();
  const char *const q_row = lds.in.q + m * QP;
  float q[NST][8];
#pragma unroll
  for (int s = 0; s < NST; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = lds.in.idx[32 * s + 8 * h + e];
      q[s][e] = c >= 0 ? E::load1(q_row, c) : 0.f;
    }
  State st;
#pragma unroll
  for (int i = 0; i < 8; ++i) st.acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  st.off[0] = st.off[1] = st.l = 0.f;
  st.m = -INFINITY;
  for (int it = wave; it < items; it += 4) {
    if (t0 + it < t1) {
      const char *const t = a.p.tile(l, b, hk, t0 + it);
      if (t != nullptr) page_tile<DT, BITS, NST>(t, a.p.lay, min(kTile, np - (t0 + it) * kTile), m, h, q, a.scale_log2, st);
    } else {
      const int r0 = (it - (t1 - t0)) * kTile;
      const size_t at = ((size_t)u * a.cap + r0) * kD * EB;
      tail_tile<DT>((const char *)a.kt + at, (const char *)a.vt + at, min(kTile, nt - r0), m, h, q_row, a.scale_log2, st);
    }
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
  const int n = tid >> 4, c0 = (tid & 15) * 8;
  if (n >= heads) return;
  float M = -INFINITY, L = 0.f, o[8] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, lds.out.ml[w][n][0]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = lds.out.ml[w][n][0], wgt = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M);
    L = fmaf(lds.out.ml[w][n][1], wgt, L);
#pragma unroll
    for (int c = 0; c < 8; ++c) o[c] = fmaf(lds.out.acc[w][n][c0 + c], wgt, o[c]);
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

template <int DT, int BITS>
hipError_t launch(const PagedDecodeArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  const int steps = (a.T + 31) / 32;
  void (*const k)(PagedDecodeArgs) = steps <= 2   ? k_paged_decode<DT, BITS, 2>
                                     : steps == 3 ? k_paged_decode<DT, BITS, 3>
                                                  : k_paged_decode<DT, BITS, 4>;
  PagedDecodeArgs copy = a;
  void *args[] = {&copy};
  hipError_t e = launch_main_kernel((const void *)k, dim3((unsigned)(a.units * a.groups * a.n_split)), dim3(256), args, 0, st);
  if (e != hipSuccess || a.n_split == 1) return e;
  hipLaunchKernelGGL(k_paged_merge<DT>, dim3((unsigned)(a.units * a.G)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace paged
}  // namespace thk
