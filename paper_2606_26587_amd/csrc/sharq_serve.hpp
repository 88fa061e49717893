// Sizes and work split of the calls around the paged cache: tables from
// request lengths, beam search's choice, and the reordering behind it.  Plain
// C++, so that a host test can replay them.
#pragma once

#include <stdint.h>

#include "sharq_kv.hpp"

namespace sharq {

// ---------------------------------------------------------------------------
// Tables from request lengths
// ---------------------------------------------------------------------------

struct AssignArgs {
  int32_t* free;
  const int32_t* count;
  int32_t *count_out, *missing;
  const int32_t *keep, *add, *held;
  int32_t *held_out, *offs, *lens, *table, *own;
  int32_t *row_seq, *positions, *slots;
  int32_t* ws;       // [2 seqs + 1]: pages given out before a sequence, columns it held; pages on the stack
  int64_t ldt;
  int pages, seqs, rows, max_len, cols, page_shift;
};

constexpr int64_t assign_workspace(int64_t seqs) { return (2 * seqs + 1) * 4; }

constexpr int kAssignThreads = 1024;
// One workgroup does it all while there is less to write than a second launch takes.
constexpr int kAssignSeqs = 2048, kAssignRows = 8192;
constexpr bool assign_whole(int64_t seqs, int64_t rows) {
  return seqs <= kAssignSeqs && (rows <= kAssignRows || seqs == 0);
}

// ---------------------------------------------------------------------------
// Beam search
// ---------------------------------------------------------------------------

constexpr int kMaxBeams = 32;
constexpr int kBeamPer = 32;                        // logits of a thread in one turn
constexpr int kBeamTile = 256 * kBeamPer;           // of a workgroup
constexpr int kBeamLists = 256;                     // candidate lists of a group: a thread each in the second kernel
constexpr int64_t kBeamLds = 56 << 10;              // what that kernel keeps in LDS at most, beside 5 KB of its own

// Bytes of LDS that joins the lists of `chunks` parts of a row: their entries, and as many candidates.
constexpr int64_t beam_lds(int64_t beams, int64_t chunks) { return beams * beams * chunks * (8 + 16); }

struct BeamSplit {
  int chunks, tiles;   // workgroups of a row of logits; their turns
};

constexpr BeamSplit beam_split(int64_t rows, int64_t beams, int64_t vocab) {
  const int64_t tiles = ceil_div(vocab, kBeamTile);
  int64_t chunks = rows > 0 ? ceil_div(1024, rows) : 1;
  if (chunks > kBeamLists / beams) chunks = kBeamLists / beams;
  if (chunks > tiles) chunks = tiles;
  while (chunks > 1 && beam_lds(beams, chunks) > kBeamLds) --chunks;
  const int64_t each = ceil_div(tiles, chunks);
  return {(int)ceil_div(tiles, each), (int)each};
}

// A wavefront's part of a row's sum: the sum of 2^((x - ref) log2 e + rest), which is that of e^x times 2^-e, where e is
// ref log2 e to the nearest whole number and rest what that leaves.
struct BeamPart {
  double sum;
  float ref;
  int32_t pad;
};

constexpr int64_t beam_lists_bytes(int64_t rows, int chunks, int64_t beams) { return rows * chunks * beams * 8; }
constexpr int64_t beam_workspace(int64_t rows, int64_t beams, int64_t vocab) {
  const BeamSplit s = beam_split(rows, beams, vocab);
  return beam_lists_bytes(rows, s.chunks, beams) + rows * s.chunks * 4 * (int64_t)sizeof(BeamPart) + 8;
}

struct BeamArgs {
  const void* logits;
  int64_t ld;
  const float* scores;
  const uint8_t* done;
  float* scores_out;
  int32_t *parents, *tokens;
  uint8_t* done_out;
  uint64_t* lists;   // [rows][chunks][beams], best first, 0: none
  BeamPart* parts;   // [rows][chunks][4]
  int beams, vocab, eos, chunks, tiles;
};

// ---------------------------------------------------------------------------
// Reordering
// ---------------------------------------------------------------------------

struct ReorderArgs {
  const int32_t *parents, *lens, *tokens;
  const int32_t* table;
  int32_t* table_out;
  int64_t ldt, ldto;
  const int32_t* ids;
  int32_t* ids_out;
  int64_t ldi, ldio;
  int32_t* copies;   // [groups * beams][3]
  int beams, cols, id_cols, page_shift;
};

// A wavefront takes 64 columns of a group's tables or ids.
constexpr int64_t reorder_units(int64_t cols) { return ceil_div(cols, 64); }

// 16-byte chunks of K and V of a page and head that a workgroup copies.
constexpr int kCopyChunks = 1024;
constexpr int copy_row_bytes(int D, int fmt) { return fmt == kKvBf16 ? 2 * D : fmt == kKvMx ? D / 2 : D; }
constexpr int64_t copy_parts(int page_size, int D, int fmt) {
  return ceil_div((int64_t)2 * page_size * copy_row_bytes(D, fmt) / 16, kCopyChunks);
}

}  // namespace sharq
