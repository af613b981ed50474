// Sums over the entries of a list that share a node: the gradient of embedding
// rows, and of keys and values that many edges read.  The list is sorted by node
// (stably, so entries of a node keep their order), then each node's entries are
// added in that order: no atomic adds into the result, and the same bits from run
// to run.
//
// Work is cut at fixed places of the sorted list, not at nodes: a group of lanes
// takes a chunk of C entries and adds every segment (the entries of one node) that
// starts in it, going on past the chunk's end where the segment ends within the next
// chunk.  A segment that reaches further is long: each of its chunks leaves a partial
// sum in 32 bits, and a second launch joins those of each long segment in order.
#pragma once

#include "dg_model.h"

namespace dg {

// A list of n IDs in [0, slots) and its stable sort.  An ID of -1 stands for no
// node; it and IDs outside [0, slots) sort behind all others as `slots`.
struct IdSort {
  const int32_t *ids;
  int64_t n, slots;
  bool compact;        // dst = rank among the distinct nodes, not the node
  // carved
  int32_t *key[2], *pos[2];  // keys and list places, alternating between passes
  int32_t *dst;        // [n] row that each sorted entry is added to: below limit(), or
                       // the entry is of no node (those are the last)
  int32_t *order;      // [n] list place of each sorted entry
  uint8_t *seen;       // [slots] whether the node occurs (!compact)
  uint32_t *cnt, *tot; // digit counts per tile, and in all
  int32_t *heads;      // distinct nodes per block of entries, then before it (compact)
  int32_t *n_long;     // long segments listed
  int32_t *long_at;    // [n / C + 1] the chunk in which each starts
  float *part;         // [2 * chunks][width] partial sums
  int32_t C;           // entries of a chunk
  int64_t chunks;
  int64_t width;       // numbers of a partial sum
  uint32_t limit() const { return compact ? 0x7fffffffu : (uint32_t)slots; }
};
// Lays the arrays out in c.
void carve_sort(IdSort &a, Carve &c);
// Bytes that lists of up to a.n entries take (tiles and chunks get longer, and their
// arrays smaller, at some lengths).
size_t sort_room(IdSort a);
// Sorts on stream s.  node_out: [n] the distinct nodes, ascending, count: how many
// (compact).  status: ORs 1 where an ID is below -1 or not below slots (optional).
int run_sort(IdSort &a, int32_t *node_out, int64_t *count, int32_t *status, hipStream_t s);

// What the group of lanes that takes chunk c does: entries [begin, stop) in order;
// a segment ends where dst changes.
struct Chunk {
  int64_t begin, stop;   // stop: the chunk's end
  int32_t last;          // dst of its last entry
  bool lead_part;        // entries from `begin` that continue a long segment
  bool trail_part;       // the last segment is long and starts here
  bool beyond;           // the last segment goes on past `stop`, into the next chunk only
};
__device__ __forceinline__ Chunk chunk_of(const int32_t *dst, int64_t n, int C, int64_t c) {
  Chunk k;
  const int64_t lo = c * C, hi = min(lo + C, n);
  // the places that decide, loaded together
  const int32_t first = dst[lo], last = dst[hi - 1];
  const int32_t before = dst[max(lo - 1, (int64_t)0)];
  const int32_t before2 = dst[max(lo - C - 1, (int64_t)0)];
  const int32_t after = dst[min(hi, n - 1)];
  const int32_t after2 = dst[min(hi + C, n - 1)];
  const bool lead = lo > 0 && before == first;
  k.begin = lo;
  k.stop = hi;
  k.last = last;
  // it starts two chunks back, or in the last one and reaches the next
  k.lead_part = lead && ((lo > C && before2 == first) || (hi < n && after == first));
  if (lead && !k.lead_part) {  // the chunk before adds these
    int64_t a = lo, b = hi;    // first entry of another segment, in (a, b]
    while (b - a > 1) {
      const int64_t m = (a + b) >> 1;
      if (dst[m] == first) a = m; else b = m;
    }
    k.begin = b;
  }
  const bool starts = !(lead && last == first);  // the last segment starts here
  const bool on = starts && hi < n && after == last;
  k.trail_part = on && hi + C < n && after2 == last;
  k.beyond = on && !k.trail_part;
  return k;
}

// Joins the partial sums of the long segments: output z (of up to two) takes columns
// at[z] .. at[z] + cols of each partial sum, times factor[z], rounded to its type.
struct JoinOut {
  void *out[2];
  int64_t stride[2];
  int64_t at[2];
  float factor[2];
};
int run_join(const IdSort &a, const JoinOut &o, int outs, int cols, int32_t type, hipStream_t s);

// Lanes per row (a power of two) and launches' column tiles for rows of `vecs`
// vectors: rows of more than 64 vectors take tiles of 64 or 32, whichever leaves
// fewer lanes idle.
struct RowLanes {
  int lg, tiles;
};
inline RowLanes row_lanes(int64_t vecs) {
  if (vecs <= 64) return {log2_up(vecs), 1};
  const int64_t t64 = (vecs + 63) / 64, t32 = (vecs + 31) / 32;
  return t32 * 32 < t64 * 64 ? RowLanes{5, (int)t32} : RowLanes{6, (int)t64};
}

}  // namespace dg
