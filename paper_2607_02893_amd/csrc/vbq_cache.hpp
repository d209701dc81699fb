// Indexes of the 4-bit cache (page layout version 1, declared in include/vbq.h): where
// a position's codes and scales lie, and which rows, positions and pages a call may
// touch.  Host code can include it, so the bounds are tested without a GPU.
#pragma once

#include <cstdint>

#include "../../include/vbq.h"

#ifdef __HIPCC__
#define VBQ_HD __host__ __device__ __forceinline__
#else
#define VBQ_HD inline
#endif

namespace vbq {

constexpr int kPage = VBQ_KV_PAGE;  // positions of a page

// Sections of one head's part of a page, in bytes from its start (D = head_dim):
// keys' codes, values' codes, keys' scales, values' scales.
template <int D>
struct PageOf {
  static constexpr int kGroups = D / 64;
  static constexpr int kKeyWords = D / 32;       // code words a lane holds of a 16-position tile
  static constexpr int kValues = 64 * D / 2;
  static constexpr int kKeyScales = 2 * kValues;
  static constexpr int kValueScales = kKeyScales + 128 * kGroups;
  static constexpr int kBytes = kValueScales + 128 * kGroups;
};

// Byte offset of the key code word that holds elements 32 j + 8 g .. + 7 of position p % 64.
template <int D>
VBQ_HD int key_word(int p, int j, int g) {
  const int lane = 16 * g + (p & 15), tile = p >> 4;
  if constexpr (D == 64) return tile * 512 + lane * 8 + j * 4;
  return tile * (64 * PageOf<D>::kKeyWords * 4) + (j >> 2) * 1024 + lane * 16 + (j & 3) * 4;
}
// Byte offset of the value code word of element d and the eight slots 8 g .. + 7 of block b.
template <int D>
VBQ_HD int value_word(int b, int d, int g) {
  return PageOf<D>::kValues + b * (16 * D) + (d >> 6) * 1024 + (16 * g + (d & 15)) * 16 + ((d >> 4) & 3) * 4;
}
VBQ_HD int slot_of(int p) { return ((p >> 2) & 3) * 8 + ((p >> 4) & 1) * 4 + (p & 3); }
// Bit offset of the i-th of a word's eight codes: pairs in the two halves, as in the packed weights.
VBQ_HD int code_bit(int i) { return 4 * (i >> 1) + 16 * (i & 1); }

// ------------------------------------------------------------------ the batch

struct Batch {
  const int32_t* table;
  const int32_t* row_start;  // null: max_rows rows a sequence
  const int32_t* seq_len;
  int32_t n_seqs, table_stride;
  int64_t n_rows;
  int32_t max_rows;
};

struct Seq {
  int64_t row0;      // its first row of the call
  int64_t n;         // its rows
  int64_t pos0;      // position of its first row (negative: rows before position 0)
  int64_t end;       // positions it has, no more than its pages hold
};

// The values of device arrays are not known to the host: whatever they are, rows stay
// within the call's rows and positions within the table's pages.
VBQ_HD Seq seq_of(const Batch& a, int b) {
  Seq s;
  int64_t r0, r1;
  if (a.row_start) {
    r0 = a.row_start[b];
    r1 = a.row_start[b + 1];
  } else {
    r0 = (int64_t)b * a.max_rows;
    r1 = r0 + a.max_rows;
  }
  r0 = r0 < 0 ? 0 : r0;
  r1 = r1 > a.n_rows ? a.n_rows : r1;
  s.row0 = r0;
  s.n = r1 > r0 ? r1 - r0 : 0;
  const int64_t len = a.seq_len[b] > 0 ? a.seq_len[b] : 0;
  const int64_t cap = (int64_t)a.table_stride * kPage;
  s.pos0 = len - s.n;
  s.end = len < cap ? len : cap;
  return s;
}

// A page's id, or -1 where the table has none of the cache's.
VBQ_HD int64_t page_id(const Batch& a, int64_t n_pages, int b, int64_t page) {
  const int32_t id = a.table[(int64_t)b * a.table_stride + page];
  return id >= 0 && (int64_t)id < n_pages ? id : -1;
}

// Workgroups that share the 32-position blocks of each head and sequence in the append and the
// read-back, each taking every so-manieth: as many as the rows need, but no more than 2^16, nor
// than makes 2^22 over all heads and sequences (with max_rows from the longest of many sequences,
// or a guess, nearly all would have nothing to do: 2^42 within the limits of a batch).
VBQ_HD int64_t blocks_of(int64_t max_rows, int64_t n_rows, int64_t heads, int64_t n_seqs) {
  const int64_t rows = max_rows < n_rows ? max_rows : n_rows;
  const int64_t blocks = (rows + 31) / 32 + (rows > 1 ? 1 : 0);  // (a row's block may begin before it)
  const int64_t share = ((int64_t)1 << 22) / (heads * n_seqs), most = share > 1 ? share : 1;
  const int64_t few = blocks < 65536 ? blocks : 65536;
  return few < most ? few : most;
}

}  // namespace vbq
