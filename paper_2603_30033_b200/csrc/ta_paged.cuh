// Paged latent KV cache: what the kernels of the paged entry points share.
//
// The pools hold pages of `page_size` consecutive slots, K [n_pages, page_size, r3] and V [n_pages, page_size, t3];
// slot i of sequence b is row i % page_size of page table[b * max_pages + i / page_size].  A table entry that a call
// needs and that is outside [0, n_pages) sets TA_DEVERR_BAD_PAGE: its rows are read as zeros, and nothing is written
// through it.  Entries that a call does not need are never looked at.
#pragma once

#include "ta_common.cuh"

namespace ta {

// Pool row of `slot` (0 <= slot < max_pages * page_size) through one sequence's table row, or -1 (flagged).
__device__ __forceinline__ long paged_row(const int32_t* __restrict__ row_table, int slot, const PagedView& pv, unsigned int* err) {
  const int j = slot / pv.page_size;
  const int pg = row_table[j];
  if (pg < 0 || pg >= pv.n_pages) {
    atomicOr(err, (unsigned)TA_DEVERR_BAD_PAGE);
    return -1;
  }
  return (long)pg * pv.page_size + (slot - j * pv.page_size);
}

// Where row `t` of a ragged batch of appended tokens goes.  tok_start [B + 1] ascending: sequence b owns the rows
// [tok_start[b], tok_start[b + 1]).  Rows at or behind tok_start[B], and in front of tok_start[0], belong to nobody.
// A token whose slot does not exist sets TA_DEVERR_BAD_CACHE_LEN and is dropped.
struct AppendDst {
  long row;      // pool row, or -1: nothing is written
  int pos;       // absolute position (angle of the rotation)
};
__device__ __forceinline__ AppendDst append_dst(int t, const int32_t* __restrict__ tok_start, const int32_t* __restrict__ cache_len,
                                                int B, int pos0, const PagedView& pv, unsigned int* err) {
  AppendDst d;
  d.row = -1; d.pos = 0;
  if (t < tok_start[0] || t >= tok_start[B]) return d;
  int lo = 0, hi = B;                       // tok_start[lo] <= t < tok_start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tok_start[mid] <= t) lo = mid; else hi = mid;
  }
  const int len = cache_len[lo];
  const long slot = (long)len + (t - tok_start[lo]);
  if (len < 0 || slot >= (long)pv.max_pages * pv.page_size) {
    atomicOr(err, (unsigned)TA_DEVERR_BAD_CACHE_LEN);
    return d;
  }
  d.pos = pos0 + (int)slot;
  d.row = paged_row(pv.table + (long)lo * pv.max_pages, (int)slot, pv, err);
  return d;
}

// Partials of a sequence, from the first and last of `grid` CTAs that the streaming kernel has noted for it; 0 where
// they cannot be its note.  (A streaming CTA whose wait ran out leaves without one, and the words hold whatever the
// workspace held: they must not become an index.)
__host__ __device__ inline int noted_parts(int first, int last, int grid) {
  return first >= 0 && first <= last && last < grid ? last - first + 1 : 0;
}

}  // namespace ta
