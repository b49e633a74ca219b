// The index arithmetic of the paged attention for the host tests: what the rows of a tile look at, range by range.
#include "mst_paged_list.h"

using mst_paged::Divider;
using mst_paged::Key;
using mst_paged::List;

extern "C" {

// info: row0, rows, t_lo, nt, p_lo, p_hi, W, N, dense; 0 where there is no such tile
int list_of(int first, int end, int len, int tokens, int group, int stride, int64_t reach, int tile, int R, int64_t* info) {
  List T;
  if (!T.locate(first, end, len, tokens, Divider::of(group), Divider::of(stride), reach, tile, R)) return 0;
  const int64_t v[9] = {T.row0, T.rows, T.t_lo, T.nt, T.p_lo, T.p_hi, (int64_t)T.W, (int64_t)T.N, T.dense};
  for (int i = 0; i < 9; ++i) info[i] = v[i];
  return 1;
}

int range_of(int first, int end, int len, int tokens, int group, int stride, int64_t reach, int tile, int R, int splits, int least,
             int split, int64_t* lo_hi_active) {
  List T;
  if (!T.locate(first, end, len, tokens, Divider::of(group), Divider::of(stride), reach, tile, R)) return -1;
  uint32_t lo = 0, hi = 0;
  int active = 0;
  const int there = T.range(splits, Divider::of(least), split, lo, hi, active);
  lo_hi_active[0] = lo;
  lo_hi_active[1] = hi;
  lo_hi_active[2] = active;
  return there;
}

// entries lo .. hi - 1: position and token; `seen` [hi - lo][nt]: which of the tile's tokens look at them
int keys_of(int first, int end, int len, int tokens, int group, int stride, int64_t reach, int tile, int R, int64_t lo, int64_t hi, int32_t* pos,
            int32_t* who, uint8_t* seen) {
  List T;
  if (!T.locate(first, end, len, tokens, Divider::of(group), Divider::of(stride), reach, tile, R)) return 0;
  for (int64_t n = lo; n < hi; ++n) {
    const Key k = T.key((uint32_t)n);
    pos[n - lo] = k.pos;
    who[n - lo] = k.who;
    for (int t = 0; t < T.nt; ++t) seen[(n - lo) * T.nt + t] = T.sees(T.p_lo + t, t, k);
  }
  return 1;
}

// many rows: first, near, far; and the range's n0, n1, m0, m1, active
int walk_of(int first, int end, int len, int tokens, int group, int stride, int64_t reach, int tile, int R, int splits, int least, int split,
            int32_t* out) {
  List T;
  if (!T.locate(first, end, len, tokens, Divider::of(group), Divider::of(stride), reach, tile, R)) return -1;
  const mst_paged::TileWalk w(T, reach);
  int r[5] = {};
  const int there = w.range(splits, least, split, r[0], r[1], r[2], r[3], r[4]);
  out[0] = w.first; out[1] = w.near; out[2] = w.far;
  for (int i = 0; i < 5; ++i) out[3 + i] = r[i];
  return there;
}
int near(int first, int end, int len, int tokens, int group, int stride, int64_t reach, int tile, int R, int p, int k) {
  List T;
  if (!T.locate(first, end, len, tokens, Divider::of(group), Divider::of(stride), reach, tile, R)) return -1;
  return mst_paged::near_sees(T.l, p, k);
}

// first, end, len; 1 where rows were left out
int rows_of(int first, int end, int len, int tokens, int32_t* out) {
  const mst_paged::RowsOf r(first, end, len, tokens);
  out[0] = r.first; out[1] = r.end; out[2] = r.len;
  return r.outside;
}

int over(uint32_t d, int n) { return Divider::of(d).over(n); }

int page(const int32_t* row, int table_stride, int page_size, int num_pages, int p, int* slot) {
  return mst_paged::page_of(row, table_stride, Divider::of(page_size), num_pages, p, *slot);
}
}
