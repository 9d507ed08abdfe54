// The paged cache's rows: written (compacted, and quantised where the pages hold codes), read back, and appended to the
// ragged tails.  Memory bounds all three: every row is read once and written once.
#include "thk_paged.h"

#include <type_traits>

namespace thk {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// A value of another lane of the 16 that share a group (a row of the wave's data paths); the control words of the moves.
template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, false));
}
constexpr int kXor8 = 0x128;    // rotation by 8
constexpr int kXor7 = 0x141;    // mirror of eight lanes
constexpr int kXor2 = 0x4e, kXor1 = 0xb1;   // permutations of four lanes
constexpr int kLane0 = 0x150;   // + n: lane n of the 16

// Extremes of two and three, as the instructions themselves: the library functions first bring every operand that is not
// known to be the result of arithmetic into canonical form, an instruction for each element.
__device__ __forceinline__ float smaller(float a, float b) { float r; asm("v_min_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b)); return r; }
__device__ __forceinline__ float larger(float a, float b) { float r; asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b)); return r; }
__device__ __forceinline__ float smaller(float a, float b, float c) { float r; asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c)); return r; }
__device__ __forceinline__ float larger(float a, float b, float c) { float r; asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c)); return r; }

// v[e], e = 0..7, each over all 16 lanes: lane m returns the extreme of v[m / 2].  Every step halves what a lane looks
// after (it hands the other half to the lane across), so that eight reductions cost 22 instructions and not 32, and what
// follows -- a group's scale and its reciprocal, some 40 instructions -- is done by two lanes for a group, not by all.
template <bool MAX>
__device__ __forceinline__ float extreme_of(const float (&v)[8], int m) {
  auto pick = [](float a, float b) { return MAX ? larger(a, b) : smaller(a, b); };
  const bool b3 = (m & 8) != 0, b2 = (m & 4) != 0, b1 = (m & 2) != 0;
  float x[4], y[2];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = pick(b3 ? v[e + 4] : v[e], from_lane<kXor8>(b3 ? v[e] : v[e + 4]));
#pragma unroll
  for (int e = 0; e < 2; ++e) y[e] = pick(b2 ? x[e + 2] : x[e], from_lane<kXor7>(b2 ? x[e] : x[e + 2]));
  // A move between lanes must not read what one of the two instructions in front of it wrote, and the compiler, which sees to
  // that for its own instructions, does not look into these: neither the result of the next step may be, nor the function's.
  float z = pick(b1 ? y[1] : y[0], from_lane<kXor2>(b1 ? y[0] : y[1]));
  asm("s_nop 1" : "+v"(z));
  z = pick(z, from_lane<kXor1>(z));
  asm("s_nop 1" : "+v"(z));
  return z;
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return (uint32_t)Elem<THK_BF16>::round_bf16(a) | ((uint32_t)Elem<THK_BF16>::round_bf16(b) << 16);
}

// Scale of a group with extremes lo, hi: its range over the number of steps, held in the element type.
template <int DT, int BITS>
__device__ __forceinline__ float group_scale(float lo, float hi) {
  const float s = (hi - lo) / (float)((1 << BITS) - 1);
  if constexpr (DT == THK_BF16) return __uint_as_float((uint32_t)Elem<THK_BF16>::round_bf16(s) << 16);
  return s;
}

// x[j][e], j = 0..3, e = 0..7: this lane's 32 elements of a group (unit j, element e).  Element e of all the group's units
// shares a scale.  ok[j] = false: unit j is written as zeros.  dst: the group's first byte; par: its eight parameters.
template <int DT, int BITS>
__device__ __forceinline__ void encode_group(const float (&x)[4][8], const bool (&ok)[4], char *dst, char *par, int m) {
  if constexpr (BITS == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == THK_BF16) {
        u32x4 u;
#pragma unroll
        for (int p = 0; p < 4; ++p)   // the elements are bf16 values: their upper halves are all there is
          u[p] = ok[j] ? (__float_as_uint(x[j][2 * p]) >> 16) | (__float_as_uint(x[j][2 * p + 1]) & 0xffff0000u) : 0u;
        st_stream((u32x4 *)(dst + (j * 16 + m) * 16), u);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 u;
#pragma unroll
          for (int p = 0; p < 4; ++p) u[p] = ok[j] ? __float_as_uint(x[j][4 * h + p]) : 0u;
          st_stream((u32x4 *)(dst + ((2 * j + h) * 16 + m) * 16), u);
        }
      }
    }
    return;
  }
  constexpr float top = (float)((1 << BITS) - 1);
  float lo8[8], hi8[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    lo8[e] = smaller(smaller(x[0][e], x[1][e], x[2][e]), x[3][e]);
    hi8[e] = larger(larger(x[0][e], x[1][e], x[2][e]), x[3][e]);
  }
  const float lo = extreme_of<false>(lo8, m), hi = extreme_of<true>(hi8, m), s = group_scale<DT, BITS>(lo, hi);
  if ((m & 1) == 0) {
    if constexpr (DT == THK_BF16) *(uint32_t *)(par + m * 2) = (__float_as_uint(s) >> 16) | (__float_as_uint(lo) & 0xffff0000u);
    else *(uint2 *)(par + m * 4) = make_uint2(__float_as_uint(s), __float_as_uint(lo));
  }
  // (x - lo) / s, correctly rounded, by Markstein's corrections of a product with the reciprocal: with r the rounded
  // 1 / s, y' = y + (t - y s) r is the rounded quotient where y is within one unit of it, which the product itself is for a
  // scale of 8 bits (no quotient of a 24-bit by an 8-bit number lies within 2^-33 of the middle of two floats, and y' is
  // within 2^-46 in front of its rounding) and one correction makes it for 24 bits.  The residuals are exact unless s is
  // near the end of the range, where the division itself is taken.  s = 0 gives r = 0 and codes 0.
  const float r = s > 0.f ? 1.f / s : 0.f;
  const bool plain = __any(s != 0.f && !(s >= 0x1p-90f && s <= 0x1p120f));
  // A quotient below 2^22 plus 1.5 * 2^23 has its nearest whole number (ties to even) in the lowest bits; codes are put
  // together with the rest of the bits in place, whose sum is taken off at the end.
  constexpr float kMagic = 0x1.8p23f;
  constexpr uint32_t kRest = 0x4b400000u;
  uint32_t word[4][BITS / 4];   // a unit per j
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int w = 0; w < BITS / 4; ++w) word[j][w] = 0;
  constexpr auto place = [](int e) { return BITS == 4 ? 4 * (e >> 1) + 16 * (e & 1) : 8 * (e & 3); };
  auto one = [&](auto divide, auto lane) {
    constexpr int e = decltype(lane)::value;
    const float le = from_lane<kLane0 + 2 * e>(lo), se = from_lane<kLane0 + 2 * e>(s), re = from_lane<kLane0 + 2 * e>(r);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float t = x[j][e] - le;
      float y;
      if constexpr (!decltype(divide)::value) {
        y = t * re;
        y = fmaf(fmaf(-y, se, t), re, y);
        if constexpr (DT == THK_F32) y = fmaf(fmaf(-y, se, t), re, y);
      } else {
        y = se > 0.f ? t / se : 0.f;
      }
      // A normal scale of 8 bits is at most 2^-8 off, and the last quotient 15.06 at most: with 4 bits it needs no bound.  A scale
      // below the normal numbers has fewer bits and may be a third off; it takes the division, and the bound.
      if constexpr (BITS == 8 || DT == THK_F32 || decltype(divide)::value) y = fminf(y, top);
      word[j][e / (32 / BITS)] += __float_as_uint(y + kMagic) << place(e);
    }
  };
  auto all = [&](auto divide) {
    one(divide, std::integral_constant<int, 0>()); one(divide, std::integral_constant<int, 1>());
    one(divide, std::integral_constant<int, 2>()); one(divide, std::integral_constant<int, 3>());
    one(divide, std::integral_constant<int, 4>()); one(divide, std::integral_constant<int, 5>());
    one(divide, std::integral_constant<int, 6>()); one(divide, std::integral_constant<int, 7>());
  };
  if (plain) all(std::true_type());
  else all(std::false_type());
  uint32_t rest = 0;
  for (int e = 0; e < 32 / BITS; ++e) rest += kRest << place(e);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int w = 0; w < BITS / 4; ++w) word[j][w] = ok[j] ? word[j][w] - rest : 0u;
  if constexpr (BITS == 4) {
    st_stream((u32x4 *)(dst + m * 16), u32x4{word[0][0], word[1][0], word[2][0], word[3][0]});
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      st_stream((u32x4 *)(dst + (k * 16 + m) * 16), u32x4{word[2 * k][0], word[2 * k][1], word[2 * k + 1][0], word[2 * k + 1][1]});
  }
}

// One block per (unit, tile of the call), or in calls that leave room for it (paged_apart) two: one for the keys, which go
// through LDS, where their kept channels are picked, and one for the values, which go straight from memory to the lane that
// encodes them.
// Bound by memory, at the rate of a copy (5.3 to 5.5 TB/s read + write): bf16 elements, 64 units x 8191 rows, 51 channels 86 us;
// 4 bits, 1024 units x 4096 rows, 76 channels 481 us.  fp32 rows of keys take 34 KB of LDS, four blocks of a compute unit: 32
// units of up to 2048 rows, 8 bits 17 us, 3.7 TB/s in its single round of blocks.
template <int DT, int BITS>
__global__ __launch_bounds__(256) void k_paged_write(PagedWriteArgs a) {
  using E = Elem<DT>;
  constexpr int EB = E::EB, PITCH = kD * EB + 16;
  __shared__ __align__(16) char rows_lds[kTile * PITCH];
  __shared__ __align__(16) int16_t idx_lds[kD];
  const int tid = threadIdx.x, m = tid & 15, grp = tid >> 4;
  const uint32_t blk = a.apart ? blockIdx.x >> 1 : blockIdx.x;   // (a grid has fewer than 2^24 blocks)
  const bool keys = !a.apart || (blockIdx.x & 1) == 0, values = !a.apart || (blockIdx.x & 1) != 0;
  const uint32_t u = a.by_tiles.of(blk), t = blk - u * (uint32_t)a.tiles;
  const UnitPlace place = a.p.place(u);
  const int b = place.b;
  const int64_t n = min((int64_t)scalar_load(a.n_rows, b), a.most);
  const int64_t row0 = a.row0 != nullptr ? scalar_load(a.row0, b) : 0;
  const int64_t r0 = (int64_t)t * kTile;
  if (r0 >= n || row0 < 0 || (row0 & (kTile - 1)) != 0) return;
  char *const dst = a.p.unit(place).tile(row0 / kTile + t);
  if (dst == nullptr) return;
  const int rows = (int)min(n - r0, (int64_t)kTile);
  const size_t base = ((size_t)u * a.src_rows + r0) * kD;   // first element of the tile's rows
  float xv[4][8], x[4][8];
  if (values) {   // lane m of group (g, q, half) takes channels 64 half + 4 m .. + 3 of its eight rows
    const int half = grp & 1, q = (grp >> 1) & 3, g = grp >> 3;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = 32 * g + 16 * (e >> 2) + 4 * q + (e & 3);
      const size_t at = base + (size_t)min(r, rows - 1) * kD + 64 * half + 4 * m;
      if constexpr (DT == THK_BF16) {
        const u32x2 w = __builtin_nontemporal_load((const u32x2 *)((const uint16_t *)a.v + at));
        xv[0][e] = __uint_as_float(w.x << 16); xv[1][e] = __uint_as_float(w.x & 0xffff0000u);
        xv[2][e] = __uint_as_float(w.y << 16); xv[3][e] = __uint_as_float(w.y & 0xffff0000u);
      } else {
        const u32x4 w = ld_stream((const u32x4 *)((const float *)a.v + at));
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[j][e] = __uint_as_float(w[j]);
      }
      if (r >= rows) xv[0][e] = xv[1][e] = xv[2][e] = xv[3][e] = 0.f;   // a group of zeros: codes and parameters are zero
    }
  }
  constexpr int CPR = kD * EB / 16;   // 16-byte pieces of a row
  if (keys) {
    for (int i = tid; i < rows * CPR; i += 256) {
      const int r = i / CPR, c = i % CPR;
      *(u32x4 *)(rows_lds + r * PITCH + c * 16) = ld_stream((const u32x4 *)((const char *)a.k + base * EB) + i);
    }
    if (tid < kD) idx_lds[tid] = tid < a.T ? a.idx[(size_t)u * a.T + tid] & (kD - 1) : 0;
  }
  if (values) {
    const bool all[4] = {true, true, true, true};
    encode_group<DT, BITS>(xv, all, dst + a.p.lay.v_codes + grp * 64 * a.p.lay.unit_bytes,
                           dst + a.p.lay.v_params + grp * 8 * 2 * EB, m);
  }
  if (!keys) return;
  __syncthreads();
  if (grp >= a.p.lay.chunks) return;
  bool ok[4];
  int channel[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) channel[e] = idx_lds[8 * grp + e];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 16 * j + m;
    ok[j] = r < rows;
    const char *const src = rows_lds + min(r, rows - 1) * PITCH;   // a row outside repeats one inside: the extremes stay
#pragma unroll
    for (int e = 0; e < 8; ++e) x[j][e] = E::load1(src, channel[e]);
    if (8 * grp + 8 > a.T) {   // past the last kept channel: zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) x[j][e] = 8 * grp + e < a.T ? x[j][e] : 0.f;
    }
  }
  encode_group<DT, BITS>(x, ok, dst + grp * 64 * a.p.lay.unit_bytes, dst + a.p.lay.k_params + grp * 8 * 2 * EB, m);
}

// The inverse of encode_group: what the lane's 32 codes stand for, rounded to fp32 (the store rounds to the element type).
template <int DT, int BITS>
__device__ __forceinline__ void decode_group(const char *src, const char *par, int m, float (&x)[4][8]) {
  constexpr int UB = BITS != 0 ? BITS : DT == THK_BF16 ? 16 : 32;
  u32x4 w[UB / 4];
#pragma unroll
  for (int k = 0; k < UB / 4; ++k) w[k] = ld_stream((const u32x4 *)(src + (k * 16 + m) * 16));
  if constexpr (BITS == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == THK_BF16) {
        Elem<DT>::unpack(w[j], x[j]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[j][e] = __uint_as_float(w[2 * j + (e >> 2)][e & 3]);
      }
    }
    return;
  }
  float s[8], lo[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (DT == THK_BF16) {
      const uint32_t p = ((const uint32_t *)par)[e];
      s[e] = __uint_as_float(p << 16);
      lo[e] = __uint_as_float(p & 0xffff0000u);
    } else {
      const float2 p = ((const float2 *)par)[e];
      s[e] = p.x;
      lo[e] = p.y;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t c;
      if constexpr (BITS == 4) c = (w[0][j] >> (4 * (e >> 1) + 16 * (e & 1))) & 15u;
      else c = (w[j >> 1][2 * (j & 1) + (e >> 2)] >> (8 * (e & 3))) & 255u;
      x[j][e] = fmaf((float)c, s[e], lo[e]);
    }
}

// One block per (unit, tile that holds rows of the call), or two as above.  Bound by memory as the write is: the cases there
// take 75 us (5.0 TB/s), 400 us (5.5) and 14 us (2.9: one round of blocks).
template <int DT, int BITS>
__global__ __launch_bounds__(256) void k_paged_read(PagedReadArgs a) {
  using E = Elem<DT>;
  constexpr int EB = E::EB;
  __shared__ __align__(16) char rows_lds[16 + kTile * kD * EB];
  const int tid = threadIdx.x, m = tid & 15, grp = tid >> 4;
  const uint32_t blk = a.apart ? blockIdx.x >> 1 : blockIdx.x;
  const bool keys = a.k_out != nullptr && (!a.apart || (blockIdx.x & 1) == 0), values = a.v_out != nullptr && (!a.apart || (blockIdx.x & 1) != 0);
  const uint32_t u = a.by_tiles.of(blk);
  const UnitPlace place = a.p.place(u);
  const int b = place.b;
  const int64_t row0 = a.row0 != nullptr ? scalar_load(a.row0, b) : 0;
  if (row0 < 0) return;
  const int64_t end = row0 + min((int64_t)scalar_load(a.n_rows, b), a.most);
  const int64_t t = row0 / kTile + (blk - u * (uint32_t)a.tiles);
  const int64_t lo = max(row0, t * kTile), hi = min(end, (t + 1) * kTile);   // rows of this block
  if (lo >= hi) return;
  const char *const src = a.p.unit(place).tile(t);
  if (src == nullptr) return;
  const size_t out_row = (size_t)u * a.out_rows + (lo - row0);
  const int first = (int)(lo - t * kTile), rows = (int)(hi - lo);
  float x[4][8];
  if (values) {
    const int half = grp & 1, q = (grp >> 1) & 3, g = grp >> 3;
    decode_group<DT, BITS>(src + a.p.lay.v_codes + grp * 64 * a.p.lay.unit_bytes, src + a.p.lay.v_params + grp * 8 * 2 * EB, m, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = 32 * g + 16 * (e >> 2) + 4 * q + (e & 3) - first;
      if (r < 0 || r >= rows) continue;
      const size_t at = (out_row + r) * kD + 64 * half + 4 * m;
      if constexpr (DT == THK_BF16) *(uint2 *)((uint16_t *)a.v_out + at) = make_uint2(bf16_pair(x[0][e], x[1][e]), bf16_pair(x[2][e], x[3][e]));
      else *(float4 *)((float *)a.v_out + at) = make_float4(x[0][e], x[1][e], x[2][e], x[3][e]);
    }
  }
  if (!keys) return;
  // The block's key rows are one run of the output.  They are put together in LDS at the output's offset from a 16-byte
  // boundary, so that whole aligned 16-byte pieces can be stored; the two ends go element by element.
  char *const dst = (char *)a.k_out + out_row * a.ld * EB;
  const int skew = (int)((uintptr_t)dst & 15);
  if (a.ld > a.T)
    for (int i = tid; i < rows * (a.ld - a.T); i += 256) {
      const int r = i / (a.ld - a.T), c = a.T + i % (a.ld - a.T);
      E::store1(rows_lds + skew, r * a.ld + c, 0.f);
    }
  if (grp < a.p.lay.chunks) {
    decode_group<DT, BITS>(src + grp * 64 * a.p.lay.unit_bytes, src + a.p.lay.k_params + grp * 8 * 2 * EB, m, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 16 * j + m - first;
      if (r < 0 || r >= rows) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * grp + e < a.T) E::store1(rows_lds + skew, r * a.ld + 8 * grp + e, x[j][e]);
    }
  }
  __syncthreads();
  const int bytes = rows * a.ld * EB;
  const int lead = min((16 - skew) & 15, bytes), whole = (bytes - lead) / 16;
  for (int i = tid; i < whole; i += 256)
    st_stream((u32x4 *)(dst + lead) + i, ((const u32x4 *)(rows_lds + skew + lead))[i]);
  const int rest = bytes - whole * 16;   // of both ends, in bytes
  for (int i = tid; i < rest / EB; i += 256) {
    const int at = i * EB < lead ? i * EB : i * EB + whole * 16;
    *(typename E::Bits *)(dst + at) = *(const typename E::Bits *)(rows_lds + skew + at);
  }
}

// One thread per 16-byte piece of a row.  4096 units, 63 rows at most of each: 33 us, 5.1 TB/s read + write; one row of each
// of 8 units 1.9 us, its launch and two trips to memory (lengths, rows).
template <int DT>
__global__ __launch_bounds__(256) void k_append_ragged(RaggedAppendArgs a) {
  constexpr int CPR = kD * Elem<DT>::EB / 16;
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(i % CPR);
  i /= CPR;
  const int r = (int)(i % a.rows);
  const int64_t u = i / a.rows;
  if (u >= a.units) return;
  const int b = (int)(u / a.N_kv % a.B);
  const int64_t src = (a.src_row0 != nullptr ? (int64_t)a.src_row0[b] : 0) + r;
  const int64_t dst = (int64_t)a.s_tail[b] + r;
  if (r >= (a.n_new != nullptr ? a.n_new[b] : 1) || src < 0 || src >= a.src_rows || dst < 0 || dst >= a.cap) return;
  const int64_t from = (u * a.src_rows + src) * CPR + c, to = (u * a.cap + dst) * CPR + c;
  ((u32x4 *)a.k_tail)[to] = ((const u32x4 *)a.k_new)[from];
  ((u32x4 *)a.v_tail)[to] = ((const u32x4 *)a.v_new)[from];
}

template <class A>
hipError_t launch(void (*k)(A), const A &a, int64_t blocks, hipStream_t st) {
  clear_stale_hip_error();
  A copy = a;
  void *args[] = {&copy};
  return launch_main_kernel((const void *)k, dim3((unsigned)blocks), dim3(256), args, 0, st);
}

}  // namespace

hipError_t launch_paged_write(int dtype, int bits, const PagedWriteArgs &a, hipStream_t st) {
  const bool f32 = dtype == THK_F32;
  return launch(bits == 0   ? (f32 ? k_paged_write<THK_F32, 0> : k_paged_write<THK_BF16, 0>)
                : bits == 4 ? (f32 ? k_paged_write<THK_F32, 4> : k_paged_write<THK_BF16, 4>)
                            : (f32 ? k_paged_write<THK_F32, 8> : k_paged_write<THK_BF16, 8>), a, a.units * a.tiles * (a.apart ? 2 : 1), st);
}
hipError_t launch_paged_read(int dtype, int bits, const PagedReadArgs &a, hipStream_t st) {
  const bool f32 = dtype == THK_F32;
  return launch(bits == 0   ? (f32 ? k_paged_read<THK_F32, 0> : k_paged_read<THK_BF16, 0>)
                : bits == 4 ? (f32 ? k_paged_read<THK_F32, 4> : k_paged_read<THK_BF16, 4>)
                            : (f32 ? k_paged_read<THK_F32, 8> : k_paged_read<THK_BF16, 8>), a,
                a.units * a.tiles * (a.apart ? 2 : 1), st);
}
hipError_t launch_paged_decode(int dtype, int bits, const PagedDecodeArgs &a, hipStream_t st) {
  return dtype == THK_F32 ? launch_paged_decode_f32(bits, a, st) : launch_paged_decode_bf16(bits, a, st);
}
hipError_t launch_append_ragged(int dtype, const RaggedAppendArgs &a, hipStream_t st) {
  const int64_t pieces = a.units * a.rows * (dtype == THK_F32 ? 32 : 16);
  return launch(dtype == THK_F32 ? k_append_ragged<THK_F32> : k_append_ragged<THK_BF16>, a, (pieces + 255) / 256, st);
}

}  // namespace thk
