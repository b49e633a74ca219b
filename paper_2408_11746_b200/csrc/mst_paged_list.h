// What a tile of query rows looks at in a paged cache: index arithmetic only, the same on the host (where it is tested, also on lengths and page
// numbers that make no sense) and on the device.
//
// A tile is up to R neighbours among one sequence's (new token, query head of one key head) pairs, so that the heads of a group share keys.
// Its keys are a list: the window of all its tokens, positions w0 .. w0 + W - 1 in order; then for each m >= 1 the positions m l behind each of its
// tokens, which only that token's rows look at.  Where a tile has l tokens or more the window is everything from 0 on and the set is left to
// the mask.  Whatever a length says, next to nothing is listed that lies at `reach` or beyond, where the table has no room for a position: the table bounds
// the work, and lists stay below 2^32 entries.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define MST_HD __host__ __device__ __forceinline__
#else
#define MST_HD inline
#endif

namespace mst_paged {

// Quotients by a number that stays, of numbers below 2^31, without a division (Granlund and Montgomery 1994: a multiplier rounded up and the quotient's
// high word, which with the number itself does not pass 32 bits)
struct Divider {
  uint32_t d, mul;
  int shift;
  static Divider of(uint32_t d) {
    int l = 0;
    while (((uint64_t)1 << l) < d) ++l;
    return Divider{d, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1), l};
  }
  MST_HD int over(int n) const {
#ifdef __CUDA_ARCH__
    return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift);
#else
    return (int)(((uint32_t)(((uint64_t)mul * (uint32_t)n) >> 32) + (uint32_t)n) >> shift);
#endif
  }
};

// The rows first .. end - 1 of a sequence that the activations' `tokens` rows have: those beyond them are cut off, positions counted from the true end
// (so a length goes down with it; below 0 nobody has a position either way).  One that starts below 0 has none, which `locate` sees to.
struct RowsOf {
  int first, end, len;
  bool outside;       // some rows, or the place of none, are not among the activations'
  MST_HD RowsOf(int first_, int end_, int len_, int tokens) : first(first_) {
    end = end_ < tokens ? end_ : tokens;
    len = len_ < 0 ? len_ : len_ - (end_ - end);
    outside = first < 0 || end_ > tokens;
  }
};

struct Key {
  int pos;    // -1: none
  int who;    // the token of the tile that alone looks at it, -1: the window
};

struct List {
  int row0, rows;         // the tile's pairs among the sequence's
  int first;              // the sequence's first row of the activations
  int t_lo, nt;           // the tokens it touches
  int p_lo, p_hi;         // their positions
  int l, w0;
  int m0;                 // the first m: 1, or what brings the tile's first token below reach
  uint32_t W, N;          // entries of the window, of the list
  bool dense;

  // Tile `tile` of `R` pairs of a sequence with rows first .. end - 1 of `tokens` and `len` positions, `group` query heads to a key head, `reach`
  // positions that its table has room for.  false: no such tile.
  MST_HD bool locate(int first_, int end, int len, int tokens, const Divider& group, const Divider& stride, int64_t reach, int tile, int R) {
    first = first_;
    l = (int)stride.d;
    if (first < 0 || end <= first || end > tokens) return false;
    const int n = end - first;
    const int64_t all = (int64_t)n * group.d, r0 = (int64_t)tile * R;
    if (r0 >= all || r0 + R > 0x7FFFFFFF) return false;
    row0 = (int)r0;
    rows = all - r0 < R ? (int)(all - r0) : R;
    t_lo = group.over(row0);
    nt = group.over(row0 + rows - 1) - t_lo + 1;
    const int64_t p = (int64_t)len - n + t_lo;
    p_lo = p < -(1 << 30) ? -(1 << 30) : (int)p;      // a length that far below its tokens: nothing is looked at either way
    p_hi = p_lo + nt - 1;
    dense = nt >= l;
    const int64_t last = p_hi < reach ? p_hi : reach - 1;
    const int64_t w = dense ? 0 : (int64_t)p_lo - l + 1;
    w0 = w > 0 ? (int)w : 0;
    W = last >= w0 ? (uint32_t)(last - w0 + 1) : 0u;
    m0 = p_lo >= reach && p_lo - reach >= l ? stride.over((int)(p_lo - reach)) : 1;
    N = W + (dense || p_hi < l ? 0u : (uint32_t)(stride.over(p_hi) - m0 + 1) * (uint32_t)nt);
    return true;
  }
  MST_HD Key key(uint32_t n) const {
    if (n < W) return Key{w0 + (int)n, -1};
    if (n >= N) return Key{-1, -1};
    uint32_t m = n - W;
    int who = 0;
    if (nt > 1) {
      const uint32_t f = m;
      m = f / (uint32_t)nt;
      who = (int)(f - m * (uint32_t)nt);
    }
    const int64_t p = (int64_t)p_lo + who - ((int64_t)m + m0) * l;
    return Key{p < 0 ? -1 : (int)p, who};
  }
  // does the row of the tile's token `t`, at position p, look at an entry
  MST_HD bool sees(int p, int t, Key k) const {
    if (k.pos < 0) return false;
    if (k.who >= 0) return k.who == t;
    const int back = p - k.pos;       // both within 2^31 of each other: positions from -2^30 on
    return back >= 0 && (back < l || (dense && back % l == 0));
  }
  // Range `split` of at most `splits` ranges of whole units of 64 entries, `least` of them at least.  active: how many ranges there are.
  MST_HD bool range(int splits, const Divider& least, int split, uint32_t& lo, uint32_t& hi, int& active) const {
    const uint32_t units = N / 64 + (N % 64 != 0 ? 1u : 0u);
    uint32_t each = least.d;
    if (splits == 1) {
      each = units;
      active = 1;
    } else if (units <= (uint64_t)each * (uint32_t)splits) {
      active = units == 0 ? 1 : least.over((int)(units - 1)) + 1;
    } else {           // longer than the launch was told
      each = units / (uint32_t)splits + (units % (uint32_t)splits != 0 ? 1u : 0u);
      active = (int)(units / each + (units % each != 0 ? 1u : 0u));
    }
    if (split >= active) return false;
    const uint64_t a = (uint64_t)each * (uint32_t)split * 64u, z = a + (uint64_t)each * 64u;
    lo = (uint32_t)a;
    hi = z < N ? (uint32_t)z : N;
    return true;
  }
};

// The same for tiles of many rows, whose keys come in tiles of 128 positions: `near` of them from `first` on with every distance 0 .. l (so the
// first strided key of every row too), then `far` steps: each row's key 2 l, 3 l, .. behind it, which no other row looks at.  Short strides
// (`dense`: 64 keys in a tile take about as long as one step) have near tiles from 0 on and no steps.  A tile whose last row has a position has one near
// tile at least.
constexpr int KEYS_OF_TILE = 128, DENSE_BELOW = 64;
struct TileWalk {
  int first, near, far, m_first;
  MST_HD TileWalk(const List& T, int64_t reach) {
    const bool dense = T.l < DENSE_BELOW;
    const int64_t from = dense || (int64_t)T.p_lo - T.l < 0 ? 0 : (int64_t)T.p_lo - T.l;
    const int64_t last = T.p_hi < reach ? T.p_hi : reach - 1;
    first = (int)(from / KEYS_OF_TILE) * KEYS_OF_TILE;
    near = T.p_hi < 0 ? 0 : last >= first ? (int)((last - first) / KEYS_OF_TILE) + 1 : 1;
    m_first = T.m0 > 2 ? T.m0 : 2;
    far = dense || T.p_hi / 2 < T.l ? 0 : T.p_hi / T.l - m_first + 1;
  }
  // Range `split` of at most `splits` equal ranges, each with `least` tiles and steps or more and a near tile: near tiles n0 .. n1 - 1, strided keys
  // m0 .. m1 - 1 steps behind.  active: how many ranges there are; with short strides over long contexts fewer than are planned for (two or three near
  // tiles and hundreds of steps: the blocks and the workspace of the others are not used).
  MST_HD bool range(int splits, int least, int split, int& n0, int& n1, int& m0, int& m1, int& active) const {
    const int64_t parts = ((int64_t)near + far + least - 1) / least;
    active = (int)(parts < splits ? parts : splits);
    if (active > near) active = near;
    if (active < 1) active = 1;
    if (split >= active) return false;
    n0 = (int)((int64_t)near * split / active);
    n1 = (int)((int64_t)near * (split + 1) / active);
    m0 = m_first + (int)((int64_t)far * split / active);
    m1 = m_first + (int)((int64_t)far * (split + 1) / active);
    return true;
  }
};
// does a row at position p look at position k of a near tile
MST_HD bool near_sees(int l, int p, int k) {
  const int back = p - k;
  return back >= 0 && (back <= l || (l < DENSE_BELOW && back % l == 0));
}

// Page of position p >= 0 in a sequence's row of the table, -1 where there is none
MST_HD int page_of(const int32_t* row, int table_stride, const Divider& page_size, int num_pages, int p, int& slot) {
  const int page = page_size.over(p);
  slot = p - page * (int)page_size.d;
  if (page >= table_stride) return -1;
  const int id = row[page];
  return id >= 0 && id < num_pages ? id : -1;
}

}  // namespace mst_paged
