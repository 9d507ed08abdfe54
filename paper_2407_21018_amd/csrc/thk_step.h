// A serving step around the paged cache: arguments of the launchers of thk_rope.hip (positions), thk_plan.hip (token map,
// page tables) and thk_beam.hip (beam search).
#pragma once
#include "thk_internal.h"
#include "thk_paged.h"

namespace thk {

// A record of the token map.
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct TokenMapArgs {
  const int32_t *n_new, *pos0, *row0;   // [B]; n_new and row0 may be nullptr (1, 0)
  int32_t *map, *starts;                // starts may be nullptr for B <= kMapSequences
  int64_t n;
  int32_t B, cap, q_rows;
};
constexpr int kMapSequences = 4096;     // whose running sums a block keeps in LDS
hipError_t launch_token_map(const TokenMapArgs &a, hipStream_t st);

struct RopeArgs {
  const void *q, *k, *v;                // any of the three may be nullptr
  void *q_out, *k_out, *v_out;
  const int32_t *map;
  const uint64_t *turns;                // 2^64ths of a turn per position, [rot / 2]
  int64_t n, ld_q, ld_k, ld_v, cap;     // n: tokens of a layer
  int32_t L, B, N_q, N_kv, q_rows, rot, layout;
  int32_t rows;                         // rows (of 128 channels) per token: those of the inputs that are there
  double gain;
};
hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t st);

struct ReserveArgs {
  const int32_t *rows, *now;            // now may be nullptr, moves then too
  int32_t *held, *table, *refs, *room, *moves;
  void *ws;
  int64_t n_pages;
  int32_t B, max_pages, page_shift;     // page_shift: log2 of a page's rows
};
constexpr int kMostSequences = 1 << 30;   // of one call
size_t reserve_ws_bytes(int64_t B);
hipError_t launch_reserve(const ReserveArgs &a, hipStream_t st);

struct PagedCopyArgs {
  PagedPool p;
  const int32_t *moves;
  int64_t n;                            // records
  int64_t units;                        // layers * KV heads
};
hipError_t launch_paged_copy(const PagedCopyArgs &a, hipStream_t st);

struct BeamArgs {
  const void *logits;
  const float *scores;
  const int32_t *done;                  // may be nullptr
  int32_t *parent, *token, *done_out;   // done_out may be nullptr
  float *score_out;
  void *ws;
  int64_t ld;
  int32_t B, W, K, V, eos;
};
size_t beam_ws_bytes(int dtype, const BeamArgs &a);   // 0: a launch would be too large
hipError_t launch_beam_select(int dtype, const BeamArgs &a, hipStream_t st);

struct ReorderArgs {
  const int32_t *parent;
  void *k_tail, *v_tail;
  int32_t *s_tail, *s_pages, *held, *table, *refs;
  int64_t prompts, n_pages;
  int32_t L, W, N_kv, ld_parent, cap, max_pages, page_shift;   // max_pages 0: no pages
};
constexpr int kMostBeams = 32, kMostContinuations = 64;
hipError_t launch_reorder(int dtype, const ReorderArgs &a, hipStream_t st);

}  // namespace thk
