// Rotary positions: queries, keys and values of new tokens to where attention and the caches read them.  Memory bounds it: every row
// is read once and written once.
#include "thk_step.h"

#include <algorithm>

namespace thk {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kTokens = 32;   // most tokens of a block

// Sine and cosine of `pos` times `turn` 2^64ths of a turn.  Whole turns fall out of the product's low 64 bits, of which the upper 32
// say where on the circle it ends (to 2^-32 of a turn); the nearest quarter turn is taken off, and the rest, within pi / 4 of
// zero, goes through the Taylor series, whose first terms left out are below 2^-29 (sine) and 2^-32 there.
__device__ __forceinline__ void turned(int pos, uint64_t turn, float gain, float &s, float &c) {
  const uint32_t at = (uint32_t)(((uint64_t)(int64_t)pos * turn) >> 32);
  const uint32_t quarter = (at + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(at - (quarter << 30)) * 0x1.921fb6p-30f;   // 2 pi / 2^32
  const float y = x * x;
  const float sn = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float cs = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
  s = gain * (quarter & 2 ? -a : a);
  c = gain * ((quarter + 1) & 2 ? -b : b);
}

// One chunk of 16 bytes back from floats, each rounded once (infinities and NaN stay what they are).
template <int DT>
__device__ __forceinline__ u32x4 packed(const float (&f)[Elem<DT>::VEC]) {
  u32x4 r;
  if constexpr (DT == THK_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{f[2 * i], f[2 * i + 1]}, bf16x2));
  }
  return r;
}

// The chunks that a lane has of a row: chunks i and i + half / VEC, pair by pair, where the halves of what is turned are whole chunks (and
// of the rest, and in the other forms, two neighbours).
enum { kHalves = 0, kPairs = 1, kHalvesAny = 2 };

// A row that a lane has a part of: where from, where to (nullptr: nowhere), which of the block's tokens, whether it is turned.
struct Row {
  const char *src;
  char *dst;
  int tok;
  bool turns;
};

// A block has `tokens` tokens (of all layers) and `part` rows of each, a row in the hands of CPR / 2 lanes of a wave.  Its sines and
// cosines are computed once, while the first rows are under way, and lie in LDS: a lane takes those of its VEC pairs for every row.
// early: rows are asked for before it is known whether they go anywhere, which spares a short call a trip to memory.
template <int DT, int FORM>
__global__ __launch_bounds__(kThreads) void k_rope(RopeArgs a, int tokens, int part, int parts, int early) {
  using E = Elem<DT>;
  constexpr int VEC = E::VEC, CPR = kD / VEC, LANES = CPR / 2, ROWS = kThreads / LANES;
  constexpr int LDR = kD + 4;
  __shared__ float sn[kTokens * 64], cs[kTokens * 64];
  __shared__ float row_lds[FORM == kHalvesAny ? ROWS * LDR : 1];
  const int tid = threadIdx.x, half = a.rot / 2;
  const int64_t group = blockIdx.x / (unsigned)parts;
  const int r0 = (int)(blockIdx.x - group * parts) * part, rows = min(part, a.rows - r0);
  const int64_t t0 = group * tokens, all = a.L * a.n;
  const int here = (int)min((int64_t)tokens, all - t0), items = here * rows;
  const int nq = a.q != nullptr ? a.N_q : 0, nk = a.k != nullptr ? a.N_kv : 0;
  const int p = tid % LANES;
  const bool split = FORM == kHalves && p < half / VEC;
  const int c0 = split ? p : 2 * p, c1 = split ? p + half / VEC : 2 * p + 1;

  auto row_of = [&](int first) {
    const int i = first + tid / LANES;
    if (i >= items) return Row{nullptr, nullptr, 0, false};
    const int tok = tokens == 1 ? 0 : i / rows, r = r0 + i - tok * rows;
    const int64_t t = t0 + tok, l = a.L == 1 ? 0 : t / a.n;
    const i32x4 rec = *(const i32x4 *)(a.map + (t - l * a.n) * 4);
    const bool is_q = r < nq, turns = r < nq + nk;
    const int h = is_q ? r : turns ? r - nq : r - nq - nk, seq = rec[0];
    const int64_t most = is_q ? a.q_rows : a.cap, row = is_q ? rec[3] : rec[2], heads = is_q ? a.N_q : a.N_kv;
    const bool packed_q = is_q && a.q_rows == 0, live = seq >= 0 && seq < a.B && (packed_q || (row >= 0 && row < most));
    char *const dst = (char *)(is_q ? a.q_out : turns ? a.k_out : a.v_out) + (packed_q ? t * heads + h : ((l * a.B + seq) * heads + h) * most + row) * kD * E::EB;
    return Row{(const char *)(is_q ? a.q : turns ? a.k : a.v) + (t * (is_q ? a.ld_q : turns ? a.ld_k : a.ld_v) + h * kD) * E::EB, live ? dst : nullptr, tok, turns};
  };
  auto load = [&](const Row &w, bool any, u32x4 &x0, u32x4 &x1) {
    if (any ? w.src != nullptr : w.dst != nullptr) {
      x0 = ld_stream((const u32x4 *)w.src + c0);
      x1 = ld_stream((const u32x4 *)w.src + c1);
    }
  };
  Row next = row_of(0);
  u32x4 n0{}, n1{};
  load(next, early != 0, n0, n1);
  for (int i = tid; i < here * 64; i += kThreads)
    if ((i & 63) < half) turned(a.map[(t0 + (i >> 6)) % a.n * 4 + 1], a.turns[i & 63], a.gain, sn[i], cs[i]);
  __syncthreads();
  for (int first = 0; first < items; first += ROWS) {
    const Row w = next;
    u32x4 x0 = n0, x1 = n1;
    if (first + ROWS < items) {
      next = row_of(first + ROWS);
      load(next, false, n0, n1);
    }
    if constexpr (FORM == kHalvesAny) {
      float f[2 * VEC];
      E::unpack(x0, (float (&)[VEC])f[0]);
      E::unpack(x1, (float (&)[VEC])f[VEC]);
      float *const mine = row_lds + tid / LANES * LDR;   // (a wave's own)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int e = 0; e < 2 * VEC; e += 4) *(float4 *)(mine + 2 * VEC * p + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (w.dst != nullptr && w.turns && 2 * VEC * p < a.rot) {
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) {
          const int c = 2 * VEC * p + e;
          const bool lower = c < half;
          const int i = min(lower ? c : c - half, 63);
          const float s = sn[w.tok * 64 + i], k = cs[w.tok * 64 + i], y = mine[min(lower ? c + half : c - half, kD - 1)];
          const float turned_e = fmaf(f[e], k, lower ? -y * s : y * s);
          f[e] = c < a.rot ? turned_e : f[e];
        }
        const u32x4 y0 = packed<DT>((const float (&)[VEC])f[0]), y1 = packed<DT>((const float (&)[VEC])f[VEC]);
        // channels that are not turned keep their bits
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          constexpr int per = VEC / 4;   // channels of a word (rot is even: a word of two has both or neither)
          x0[u] = 2 * VEC * p + u * per < a.rot ? y0[u] : x0[u];
          x1[u] = 2 * VEC * p + VEC + u * per < a.rot ? y1[u] : x1[u];
        }
      }
    } else if (w.dst != nullptr && w.turns && p * VEC < half) {
      float f0[VEC], f1[VEC];
      E::unpack(x0, f0);
      E::unpack(x1, f1);
      const float *const s = sn + w.tok * 64 + p * VEC, *const k = cs + w.tok * 64 + p * VEC;
      if constexpr (FORM == kHalves) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float x = f0[e], y = f1[e];
          f0[e] = fmaf(x, k[e], -y * s[e]);
          f1[e] = fmaf(y, k[e], x * s[e]);
        }
        x0 = packed<DT>(f0);
        x1 = packed<DT>(f1);
      } else {
        const u32x4 was0 = x0, was1 = x1;
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const int h = e / 2, g = (VEC + e) / 2;   // pairs of the two chunks
          float x = f0[e], y = f0[e + 1];
          f0[e] = fmaf(x, k[h], -y * s[h]);
          f0[e + 1] = fmaf(y, k[h], x * s[h]);
          x = f1[e], y = f1[e + 1];
          f1[e] = fmaf(x, k[g], -y * s[g]);
          f1[e + 1] = fmaf(y, k[g], x * s[g]);
        }
        x0 = packed<DT>(f0);
        x1 = packed<DT>(f1);
        if (p * VEC + VEC > half) {   // pairs behind the last one keep their bits
          constexpr int per = VEC / 4;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (2 * VEC * p + u * per >= a.rot) x0[u] = was0[u];
            if (2 * VEC * p + VEC + u * per >= a.rot) x1[u] = was1[u];
          }
        }
      }
    }
    if (w.dst != nullptr) {
      st_stream((u32x4 *)w.dst + c0, x0);
      st_stream((u32x4 *)w.dst + c1, x1);
    }
  }
}

template <int DT>
const void *kernel_of(const RopeArgs &a) {
  if (a.layout == THK_ROPE_PAIRS) return (const void *)k_rope<DT, kPairs>;
  return a.rot / 2 % Elem<DT>::VEC == 0 ? (const void *)k_rope<DT, kHalves> : (const void *)k_rope<DT, kHalvesAny>;
}

}  // namespace

// Large calls: all rows of some tokens a block.  Small ones, which would leave compute units without a block: the rows of one
// pass.
hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  RopeArgs copy = a;
  const int pass = dtype == THK_F32 ? 16 : 32;
  const int64_t all = a.L * a.n;
  const bool large = all * a.rows >= (int64_t)pass * 16 * kCUs;
  int tokens = large ? std::min(std::max(4 * pass / a.rows, 1), kTokens) : 1;
  int part = large ? a.rows : std::min(pass, a.rows), parts = (a.rows + part - 1) / part, early = all * a.rows <= 4 * pass * kCUs;
  void *args[] = {&copy, &tokens, &part, &parts, &early};
  return launch_main_kernel(dtype == THK_F32 ? kernel_of<THK_F32>(a) : kernel_of<THK_BF16>(a),
                            dim3((unsigned)((all + tokens - 1) / tokens * parts)), dim3(kThreads), args, 0, st);
}

}  // namespace thk
