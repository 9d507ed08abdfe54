// Rotary positions: queries, keys and values of new tokens to where attention and the caches read them.  Memory bounds it: every row
// is read once and written once (16384 tokens of 64 + 16 heads, bf16: 671 MB in 115 us, 5.8 TB/s); small calls a launch and two trips (one token: 3.0 us).
#include "thk_step.h"

#include <algorithm>

namespace thk {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;

// Sine and cosine of `pos` times `turn` 2^64ths of a turn, times the gain, rounded once.  Whole turns fall out of the product's low 64 bits, of which
// the upper 32 say where on the circle it ends (to 2^-32 of a turn); the nearest quarter turn is taken off, and the rest, within pi / 4
// of zero, goes through the Taylor series in 64 bits, whose first terms left out are below 2^-37 (sine) and 2^-33 there.  They are computed once for all
// of a token's rows, behind the first rows' loads (against 32 bits: one token 2.96 -> 3.04 us, longer calls the same).
__device__ __forceinline__ void turned(int pos, uint64_t turn, double gain, float &s, float &c) {
  const uint32_t at = (uint32_t)(((uint64_t)(int64_t)pos * turn + 0x80000000u) >> 32);
  const uint32_t quarter = (at + 0x20000000u) >> 30;
  const double x = (double)(int32_t)(at - (quarter << 30)) * 0x1.921fb54442d18p-30;   // 2 pi / 2^32
  const double y = x * x;
  const double sn = fma(x * y, fma(y, fma(y, fma(y, fma(y, -1. / 39916800, 1. / 362880), -1. / 5040), 1. / 120), -1. / 6), x);
  const double cs = fma(y, fma(y, fma(y, fma(y, fma(y, -1. / 3628800, 1. / 40320), -1. / 720), 1. / 24), -0.5), 1.);
  const double a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
  s = (float)(gain * (quarter & 2 ? -a : a));
  c = (float)(gain * ((quarter + 1) & 2 ? -b : b));
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

// How a row's pairs lie in its chunks of 16 bytes: in chunks i and i + half / VEC, where the halves of what is turned are whole chunks; inside
// a chunk; anyhow.
enum { kHalves = 0, kPairs = 1, kHalvesAny = 2 };
constexpr int most_tokens(int form) { return form == kHalvesAny ? 8 : 32; }   // of a block: 8 or 16 KB of sines and cosines

// A block has `tokens` tokens (of all layers) and `part` rows of each, a row in the hands of CPR / 2 lanes of a wave.  Its sines and
// cosines are computed once, while the first rows are under way, and lie in LDS: a lane takes those of its VEC pairs for every row.  Rows are
// asked for a pass ahead, and nothing in the loop waits for memory but they (a wait for a load is one for all stores in front of it too).
// The first rows are asked for before it is known whether they go anywhere, which spares a trip to memory, but for queries of which
// few are kept (early: those too).  pick: a block's keys and values come first, then the queries that are kept.
// kHalvesAny has a sine and a cosine for each channel, and the channels' mates change places through LDS.
template <int DT, int FORM>
__global__ __launch_bounds__(kThreads, 6) void k_rope(RopeArgs a, int tokens, int part, int parts, int early, int pick) {
  using E = Elem<DT>;
  constexpr int VEC = E::VEC, CPR = kD / VEC, LANES = CPR / 2, ROWS = kThreads / LANES;
  constexpr bool ANY = FORM == kHalvesAny;
  constexpr int ANGLES = ANY ? kD : 64, LDR = kD + 4;
  __shared__ __align__(16) float sn[most_tokens(FORM) * ANGLES], cs[most_tokens(FORM) * ANGLES];
  __shared__ __align__(16) float mates[ANY ? ROWS * LDR : 4];
  __shared__ i32x4 records[most_tokens(FORM)];
  __shared__ int kept[most_tokens(FORM)], n_kept;   // pick: the tokens whose queries go somewhere
  const int tid = threadIdx.x, half = a.rot / 2;
  const int64_t group = blockIdx.x / (unsigned)parts;
  const int r0 = (int)(blockIdx.x - group * parts) * part, rows = min(part, a.rows - r0);
  // (pick: tokens as far apart as there are blocks, so that those whose queries are kept, a sequence's last, are spread over the blocks)
  const int64_t all = a.L * a.n, apart = pick ? gridDim.x : 1, t0 = pick ? group : group * tokens;
  const int here = (int)min((int64_t)tokens, (all - t0 + apart - 1) / apart);
  const int nv = a.v != nullptr ? a.N_kv : 0, nk = a.k != nullptr ? a.N_kv : 0;   // rows of a token: values, keys, queries
  const int p = tid % LANES;
  // (neighbouring lanes have neighbouring chunks in both loads and both stores)
  const int c0 = FORM != kHalves || p < half / VEC ? p : p + half / VEC, c1 = FORM == kHalves && p < half / VEC ? p + half / VEC : p + LANES;

  struct Place { int tok, r; };   // token and row of what a lane has in the pass that begins at `first`
  const int others = here * (nv + nk);   // pick: these come first
  int items = pick ? others : here * rows;
  auto place = [&](int first) {
    int i = min(first + tid / LANES, items - 1);
    const bool is_q = pick && i >= others;
    const int each = pick ? is_q ? a.N_q : nv + nk : rows;
    i -= is_q ? others : 0;
    const int t = tokens == 1 ? 0 : i / each;
    return Place{is_q ? kept[t] : t, r0 + i - t * each + (is_q ? nv + nk : 0)};
  };
  auto source = [&](const Place &w) {
    const bool is_q = w.r >= nv + nk, turns = w.r >= nv;
    const int h = is_q ? w.r - nv - nk : turns ? w.r - nv : w.r;
    return (const u32x4 *)((const char *)(is_q ? a.q : turns ? a.k : a.v) + ((t0 + w.tok * apart) * (is_q ? a.ld_q : turns ? a.ld_k : a.ld_v) + h * kD) * E::EB);
  };
  auto target = [&](const Place &w, int first) -> u32x4 * {   // nullptr: nowhere
    const i32x4 rec = records[w.tok];
    const bool is_q = w.r >= nv + nk, turns = w.r >= nv;
    const int h = is_q ? w.r - nv - nk : turns ? w.r - nv : w.r, seq = rec[0];
    const int64_t t = t0 + w.tok * apart, l = a.L == 1 ? 0 : t / a.n;
    const int64_t most = is_q ? a.q_rows : a.cap, row = is_q ? rec[3] : rec[2], heads = is_q ? a.N_q : a.N_kv;
    const bool packed_q = is_q && a.q_rows == 0;
    if (first + tid / LANES >= items || seq < 0 || seq >= a.B || (!packed_q && (row < 0 || row >= most))) return nullptr;
    return (u32x4 *)((char *)(is_q ? a.q_out : turns ? a.k_out : a.v_out) + (packed_q ? t * heads + h : ((l * a.B + seq) * heads + h) * most + row) * kD * E::EB);
  };

  const uint64_t turn = (tid & 63) < half ? a.turns[tid & 63] : 0;
  if (tid < here) {
    const int64_t t = t0 + tid * apart;
    const i32x4 r = *(const i32x4 *)(a.map + (a.L == 1 ? t : t % a.n) * 4);
    records[tid] = r;
    if (pick) {   // (fewer tokens than a wave's lanes)
      const bool keep = r[0] >= 0 && r[0] < a.B && r[3] >= 0 && r[3] < a.q_rows;
      const unsigned long long m = __ballot(keep);
      if (keep) kept[__popcll(m & ((1ull << tid) - 1))] = tid;
      if (tid == 0) n_kept = __popcll(m);
    }
  }
  Place now = place(0);
  u32x4 n0{}, n1{};
  const bool sure = pick ? tid / LANES < others : early || now.r < nv + nk || a.q_rows == 0;
  if (sure) {
    const u32x4 *const x = source(now);
    n0 = ld_stream(x + c0);
    n1 = ld_stream(x + c1);
  }
  __syncthreads();
  if (pick) {
    items = others + n_kept * a.N_q;
    now = place(0);
  }
  u32x4 *to = target(now, 0);
  if (!sure && to != nullptr) {
    const u32x4 *const x = source(now);
    n0 = ld_stream(x + c0);
    n1 = ld_stream(x + c1);
  }
  for (int i = tid; i < here * 64; i += kThreads) {   // (kThreads is a multiple of 64)
    const int tok = i >> 6, j = i & 63;
    float s, c;
    turned(records[tok][1], turn, a.gain, s, c);
    if constexpr (ANY) {
      if (j < half) {
        sn[tok * kD + j] = -s;
        sn[tok * kD + j + half] = s;
        cs[tok * kD + j] = cs[tok * kD + j + half] = c;
      }
    } else {
      sn[i] = s;
      cs[i] = c;
    }
  }
  __syncthreads();
  for (int first = 0; first < items; first += ROWS) {
    u32x4 x0 = n0, x1 = n1, *const dst = to;
    const int tok = now.tok;
    const bool turns = dst != nullptr && now.r >= nv;
    if (first + ROWS < items) {
      now = place(first + ROWS);
      to = target(now, first + ROWS);
      if (to != nullptr) {
        const u32x4 *const x = source(now);
        n0 = ld_stream(x + c0);
        n1 = ld_stream(x + c1);
      }
    }
    if constexpr (ANY) {
      float *const row = mates + tid / LANES * LDR;   // (a wave's own)
      auto give = [&](const u32x4 &x, int c) {   // the chunk's elements to where their mates look for them
        if (c >= a.rot) return;
        float f[VEC];
        E::unpack(x, f);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (c + e < a.rot) row[c + e < half ? c + e + half : c + e - half] = f[e];
      };
      auto turn_chunk = [&](u32x4 &x, int c) {
        if (!turns || c >= a.rot) return;
        float f[VEC];
        E::unpack(x, f);
        const float *const s = sn + tok * kD + c, *const k = cs + tok * kD + c, *const y = row + c;
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = fmaf(f[e], k[e], y[e] * s[e]);
        const u32x4 z = packed<DT>(f);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = c + u * (VEC / 4) < a.rot ? z[u] : x[u];   // channels that are not turned keep their bits (rot is even: a word of two has both or neither)
      };
      give(x0, c0 * VEC);
      give(x1, c1 * VEC);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      turn_chunk(x0, c0 * VEC);
      __builtin_amdgcn_sched_barrier(0);   // (one chunk's operands in registers at a time)
      turn_chunk(x1, c1 * VEC);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else if constexpr (FORM == kHalves) {
      if (turns && p * VEC < half) {
        float f0[VEC], f1[VEC];
        E::unpack(x0, f0);
        E::unpack(x1, f1);
        const float *const s = sn + tok * 64 + p * VEC, *const k = cs + tok * 64 + p * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float x = f0[e], y = f1[e];
          f0[e] = fmaf(x, k[e], -y * s[e]);
          f1[e] = fmaf(y, k[e], x * s[e]);
        }
        x0 = packed<DT>(f0);
        x1 = packed<DT>(f1);
      }
    } else {
      auto turn_chunk = [&](u32x4 &x, int c) {   // c: its first channel
        if (!turns || c >= a.rot) return;
        float f[VEC];
        E::unpack(x, f);
        const float *const s = sn + tok * 64 + c / 2, *const k = cs + tok * 64 + c / 2;
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const float u = f[e], v = f[e + 1];
          f[e] = fmaf(u, k[e / 2], -v * s[e / 2]);
          f[e + 1] = fmaf(v, k[e / 2], u * s[e / 2]);
        }
        const u32x4 z = packed<DT>(f);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = c + u * (VEC / 4) < a.rot ? z[u] : x[u];   // pairs behind the last one keep their bits
      };
      turn_chunk(x0, c0 * VEC);
      turn_chunk(x1, c1 * VEC);
    }
    if (dst != nullptr) {
      st_stream(dst + c0, x0);
      st_stream(dst + c1, x1);
    }
  }
}

template <int DT>
const void *kernel_of(int form) {
  return form == kPairs ? (const void *)k_rope<DT, kPairs> : form == kHalves ? (const void *)k_rope<DT, kHalves> : (const void *)k_rope<DT, kHalvesAny>;
}

}  // namespace

// Large calls: all rows of some tokens a block.  Small ones, which would leave compute units without a block: the rows of one
// pass.  Large ones that keep a third of the queries at most (pick; of a half it gains nothing): a pass of the rows that go somewhere.
// 2048 tokens of 32 + 16 rows bf16, 32 a sequence kept: 9.1 us, all rows a block 9.6 (a part of the head) and 9.2 (whole); 16384 tokens 30 and 41;
// 49296 of 7 + 2 fp32: 25 and 47; 1950 of 160 + 80: 59 and 63.  With two passes a block 11, 33, 26 and 59.
hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t st) {
  clear_stale_hip_error();
  RopeArgs copy = a;
  const int pass = dtype == THK_F32 ? 16 : 32;
  const int64_t all = a.L * a.n;
  const int form = a.layout == THK_ROPE_PAIRS ? kPairs : a.rot / 2 % (dtype == THK_F32 ? 4 : 8) == 0 ? kHalves : kHalvesAny;
  const bool large = all >= 2 * kCUs;
  int tokens = large ? std::min(std::max(2 * pass / a.rows, 1), most_tokens(form)) : 1;
  int part = large ? a.rows : std::min(pass, a.rows), parts = (a.rows + part - 1) / part, early = all * a.rows <= 4 * pass * kCUs;
  const int64_t kv = ((a.k != nullptr) + (a.v != nullptr)) * (int64_t)a.N_kv, most_q = (int64_t)a.B * a.q_rows;
  int pick = large && a.q != nullptr && kv > 0 && a.q_rows > 0 && 3 * most_q <= a.n;
  if (pick) {
    const int64_t each = kv + a.N_q * most_q / a.n;   // rows of a token that go somewhere
    tokens = (int)std::min<int64_t>(std::max<int64_t>((pass + each / 2) / each, 1), most_tokens(form));
  }
  void *args[] = {&copy, &tokens, &part, &parts, &early, &pick};
  return launch_main_kernel(dtype == THK_F32 ? kernel_of<THK_F32>(form) : kernel_of<THK_BF16>(form),
                            dim3((unsigned)((all + tokens - 1) / tokens * parts)), dim3(kThreads), args, 0, st);
}

}  // namespace thk
