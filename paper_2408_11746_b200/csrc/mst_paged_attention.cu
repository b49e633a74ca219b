// Attention of new tokens over a paged cache, the serving form of the strided attention:
//   Out = sum_{j in S_i} softmax_j(q . k_j / sqrt(d)) v_j,   S_i = { j <= i : i - j < l  or  (i - j) mod l == 0 }.
// Tiles of rows and the lists of keys they look at: mst_paged_list.h.  Few rows (one token, drafts): paged_rows_kernel, a block per (tile, key head,
// sequence, range of the list).
#include "mst_paged_attention.cuh"

namespace {
using namespace mst_paged;
using mst_att::ldsm_x4;
using mst_att::ldsm_x4_t;
using mst_att::mma_bf16;

// how many entries below `f` of the list behind the window are token `t`'s of `nt`
__device__ __forceinline__ uint32_t steps_below(uint32_t f, uint32_t t, uint32_t nt) { return f > t ? (f - t - 1) / nt + 1 : 0u; }

// ---------------------------------------------------------------------------------------------- few rows
// Four warps go through a range of the list, each through every fourth step of it with a ring of its own (no block-wide step until the
// end): K and V rows of a step come in by 16-byte asynchronous copies, two steps ahead, and where they are is looked up a step before that.
// Products are warp-level with the keys as the 16 rows of the left operand, S^T = K Q^T and O^T = V^T P^T, so that queries come in eights:
// of the few there are, none pays for more than seven that are not there.  The warps' softmaxes are joined through shared memory, ranges by a second
// launch.  Bound: chains of dependent instructions where lists are short (a step of 32 keys takes a warp 1100 clocks alone and 1900 with another one),
// HBM where they are long: one token each of 16 sequences over 1500 to 32768 positions, 20 heads on 4, 38 us (174 MB; queries on the left in
// sixteens, page numbers asked for where they are used: 59).
constexpr int RW = 4;             // warps
constexpr int RING = 3;
constexpr float MOST = 65536.f;   // weights of a step that add up to more ask for a new reference
template <int D>
struct RowsShape {
  static constexpr int KEYS = 2048 / D;                   // of a step: 32 or 16
  static constexpr int STEP_BYTES = KEYS * D * 2;         // 4 KiB each of K and V
  static constexpr int WARP_BYTES = RING * 2 * STEP_BYTES;
  static constexpr int SMEM = RW * WARP_BYTES + 128;
};
// 16-byte piece of a row of D values, rows D * 2 bytes apart
template <int D>
__device__ __forceinline__ uint32_t piece(uint32_t base, int row, int p) {
  return base + (uint32_t)(row * D * 2) + (((uint32_t)p ^ (uint32_t)(row & 7)) << 4);
}
// an 8 x 8 matrix of 16-bit values spread over the warp, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t t;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
  return t;
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * RW, 2) paged_rows_kernel(const __grid_constant__ Params P) {
  constexpr int R = 8 * NT, KEYS = RowsShape<D>::KEYS, STEP = RowsShape<D>::STEP_BYTES, PIECES = D / 8, AT_ONCE = 32 / PIECES, G16 = KEYS / 16;
  extern __shared__ unsigned char smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = lane & 3, mrow = lane >> 2;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  // heads first: blocks that run side by side read neighbouring rows of the same pages
  const int kvh = (int)blockIdx.x % P.C.kv_heads, split = (int)blockIdx.x / P.C.kv_heads, b = blockIdx.z;
  const uint32_t ring = ((smem_u32(smem_raw) + 127u) & ~127u) + (uint32_t)(warp * RowsShape<D>::WARP_BYTES);
  float* join = reinterpret_cast<float*>(smem_raw + (((smem_u32(smem_raw) + 127u) & ~127u) - smem_u32(smem_raw)));
  __shared__ float stat[RW][R][2];
  for (int tile = blockIdx.y;; tile += gridDim.y) {
    List T;
    if (!locate(T, P, b, tile, R)) return;
    uint32_t lo, hi;
    int active;
    if (!T.range(P.splits, P.by_least, split, lo, hi, active)) continue;
    const uint32_t total = (hi - lo + KEYS - 1) / KEYS;                                // steps of the block
    const uint32_t mine = total > (uint32_t)warp ? (total - warp + RW - 1) / RW : 0u;
    // Step s of this warp: entries lo + (s RW + warp) KEYS ..; places in the cache are numbers of 16-byte pieces.
    // An entry's page is asked for RING steps before its number is used: a warp stands still where it uses what has not come.
    Key keys[RING];
    bool seen[RING];                  // every row sees every entry of the step
    struct Entry { Key key; int slot, id; };
    const uint32_t head_at = (uint32_t)((int64_t)kvh * P.C.head_stride / 8), page_step = (uint32_t)(P.C.page_stride / 8), slot_step = (uint32_t)(P.C.token_stride / 8);
    const int32_t* table = P.B.table + (int64_t)b * P.B.table_stride;
    auto look = [&](uint32_t s) {
      const uint64_t n = (uint64_t)lo + ((uint64_t)s * RW + warp) * KEYS + lane % KEYS;
      Entry e = {n < hi ? T.key((uint32_t)n) : Key{-1, -1}, 0, -1};
      if (e.key.pos >= 0) {
        const int page = P.C.by_page.over(e.key.pos);
        e.slot = e.key.pos - page * P.C.page_size;
        if (page < P.B.table_stride) e.id = __ldg(table + page);
      }
      return e;
    };
    // Addresses that a lane comes back to; what else there is to them (slot, sixteen, row) is a constant of the unrolled loop.  Swizzle: 16-byte
    // piece p of row r at p ^ (r & 7).
    const int c = lane % PIECES, r_in = lane / PIECES;
    constexpr int SAME = 8 / AT_ONCE;       // copies whose rows take turns in the swizzle
    uint32_t to[SAME];
#pragma unroll
    for (int i = 0; i < SAME; ++i) to[i] = piece<D>(ring, i * AT_ONCE + r_in, c);
    const __nv_bfloat16 *from_k = P.C.K + c * 8, *from_v = P.C.V + c * 8;
    uint32_t frag_k[D / 16], frag_v[D / 16];
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      frag_k[k] = piece<D>(ring, lane & 15, k * 2 + (lane >> 4));
      frag_v[k] = piece<D>(ring + STEP, (lane & 7) + (lane >> 4) * 8, k * 2 + ((lane >> 3) & 1));
    }
    auto load = [&](int slot, Entry e) {
      const bool there = e.key.pos >= 0 && (uint32_t)e.id < (uint32_t)P.C.num_pages;
      if (e.key.pos >= 0 && !there) {
        e.key.pos = -1;
        g_bad_page = 1;
      }
      const uint32_t at = there ? (uint32_t)e.id * page_step + (uint32_t)e.slot * slot_step + head_at : 0u;
      const uint32_t bits = __ballot_sync(0xffffffffu, there) >> r_in;
      keys[slot] = e.key;
      seen[slot] = __all_sync(0xffffffffu, e.key.pos >= 0 && (e.key.who >= 0 ? T.nt == 1 : e.key.pos <= T.p_lo && T.p_hi - e.key.pos < T.l));
#pragma unroll
      for (int r0 = 0; r0 < KEYS; r0 += AT_ONCE) {
        const uint32_t a = __shfl_sync(0xffffffffu, at, r0 + r_in);
        const uint32_t size = ((bits >> r0) & 1u) << 4;
        const uint32_t dst = to[(r0 / AT_ONCE) % SAME] + (uint32_t)(slot * 2 * STEP + r0 / 8 * 8 * D * 2);
        cp16_of(dst, from_k + (uint64_t)a * 8, size);
        cp16_of(dst + STEP, from_v + (uint64_t)a * 8, size);
      }
    };
    Entry ahead[RING];                // of the steps to be loaded next
    {
      Entry first[RING - 1];
#pragma unroll
      for (int s = 0; s < RING - 1; ++s) first[s] = look((uint32_t)s);
#pragma unroll
      for (int s = RING - 1; s < 2 * RING - 1; ++s) ahead[s % RING] = look((uint32_t)s);
#pragma unroll
      for (int s = 0; s < RING - 1; ++s) {
        if ((uint32_t)s < mine) load(s, first[s]);
        cp_commit();
      }
    }
    // queries: the right operand's published layout (column lane / 4, rows 2 (lane % 4) and + 8)
    uint32_t q[NT][D / 16][2];
    int pos[NT][2], tok[NT][2];     // of the rows whose scores the lane holds: 2 (lane % 4) and the next
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = nt * 8 + 2 * col + u;
        const int t = P.by_group.over(T.row0 + (r < T.rows ? r : 0));
        tok[nt][u] = t - T.t_lo;
        pos[nt][u] = T.p_lo + tok[nt][u];
      }
      const int r = nt * 8 + mrow, at = T.row0 + (r < T.rows ? r : 0), t = P.by_group.over(at), h = kvh * P.group + at - t * P.group;
      const uint32_t* src = reinterpret_cast<const uint32_t*>(P.Q + (int64_t)(T.first + t) * P.ldq + (int64_t)h * D) + col;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        q[nt][k][0] = src[k * 8];
        q[nt][k][1] = src[k * 8 + 4];
      }
    }
    float acc[NT][D / 16][4], m[NT][2], sum[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int d = 0; d < D / 16; ++d) acc[nt][d][0] = acc[nt][d][1] = acc[nt][d][2] = acc[nt][d][3] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      sum[nt][0] = sum[nt][1] = 0.f;
    }
    for (uint32_t s0 = 0; s0 < mine; s0 += RING) {
#pragma unroll
      for (int slot = 0; slot < RING; ++slot) {
        const uint32_t s = s0 + slot;
        if (s >= mine) break;
        cp_wait<RING - 2>();
        __syncwarp();                      // every lane's copies are in, and the slot to be filled has been read by every lane
        if (s + RING - 1 < mine) {
          load((slot + RING - 1) % RING, ahead[(slot + RING - 1) % RING]);
          ahead[(slot + RING - 1) % RING] = look(s + 2 * RING - 1);
        }
        cp_commit();
        float x[NT][G16][4], p[NT][G16][4];      // scores and weights: keys lane / 4 and + 8 of each sixteen, rows 2 (lane % 4) and the next
#pragma unroll
        for (int g = 0; g < G16; ++g) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) x[nt][g][0] = x[nt][g][1] = x[nt][g][2] = x[nt][g][3] = 0.f;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            uint32_t f[4];
            ldsm_x4(f, frag_k[k] + (uint32_t)(slot * 2 * STEP + g * 16 * D * 2));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16(x[nt][g], f, q[nt][k][0], q[nt][k][1]);
          }
        }
        const Key key = keys[slot];
        if (!seen[slot]) {
#pragma unroll
          for (int g = 0; g < G16; ++g)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int from = g * 16 + 8 * e + mrow;
              const Key k = {__shfl_sync(0xffffffffu, key.pos, from), __shfl_sync(0xffffffffu, key.who, from)};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                  if (!T.sees(pos[nt][u], tok[nt][u], k)) x[nt][g][2 * e + u] = -INFINITY;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // Weights against the reference as it is.  Their sums tell whether a score lies too far above it, which is seldom: nobody waits for a maximum
          float add[2];
          auto weigh = [&]() {
            const float r0 = reference(m[nt][0]), r1 = reference(m[nt][1]);
            add[0] = add[1] = 0.f;
#pragma unroll
            for (int g = 0; g < G16; ++g) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                p[nt][g][2 * e] = ex2(fmaf(x[nt][g][2 * e], P.scale_log2, -r0));
                p[nt][g][2 * e + 1] = ex2(fmaf(x[nt][g][2 * e + 1], P.scale_log2, -r1));
              }
              add[0] += p[nt][g][0] + p[nt][g][2];
              add[1] += p[nt][g][1] + p[nt][g][3];
            }
          };
          weigh();
          if (__any_sync(0xffffffffu, add[0] > MOST || add[1] > MOST || m[nt][0] == -INFINITY || m[nt][1] == -INFINITY)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              float top = -INFINITY;
#pragma unroll
              for (int g = 0; g < G16; ++g) top = fmaxf(top, fmaxf(x[nt][g][u], x[nt][g][2 + u]));
              top *= P.scale_log2;
#pragma unroll
              for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              const bool up = top > m[nt][u];            // the same in all lanes of a row
              const float c = up ? ex2(m[nt][u] - top) : 1.f;
              if (up) m[nt][u] = top;
              sum[nt][u] *= c;
#pragma unroll
              for (int d = 0; d < D / 16; ++d) {
                acc[nt][d][u] *= c;
                acc[nt][d][2 + u] *= c;
              }
            }
            weigh();
          }
          sum[nt][0] += add[0];
          sum[nt][1] += add[1];
        }
#pragma unroll
        for (int g = 0; g < G16; ++g) {
          uint32_t w[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            w[nt][0] = transposed(pack_bf16(p[nt][g][0], p[nt][g][1]));
            w[nt][1] = transposed(pack_bf16(p[nt][g][2], p[nt][g][3]));
          }
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            uint32_t f[4];
            ldsm_x4_t(f, frag_v[d] + (uint32_t)(slot * 2 * STEP + g * 16 * D * 2));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16(acc[nt][d], f, w[nt][0], w[nt][1]);
          }
        }
      }
    }
    cp_wait<0>();
    // the warps' softmaxes meet in the rings' place
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = nt * 8 + 2 * col + u;
        float v = sum[nt][u];
#pragma unroll
        for (int d = 4; d < 32; d *= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (mrow == 0) {
          stat[warp][r][0] = m[nt][u];
          stat[warp][r][1] = v;
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          join[(warp * R + r) * D + d * 16 + mrow] = acc[nt][d][u];
          join[(warp * R + r) * D + d * 16 + 8 + mrow] = acc[nt][d][2 + u];
        }
      }
    static_assert(RW * R * D * 4 <= RowsShape<D>::SMEM - 128, "the sums fit the rings");
    __syncthreads();
    constexpr int E = D / 32;
    for (int r = warp; r < T.rows; r += RW) {
      float mm = -INFINITY, total_w = 0.f, o[E];
#pragma unroll
      for (int w = 0; w < RW; ++w) mm = fmaxf(mm, stat[w][r][0]);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
      for (int w = 0; w < RW; ++w) {
        const float c = ex2(stat[w][r][0] - reference(mm));
        total_w = fmaf(c, stat[w][r][1], total_w);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(c, join[(w * R + r) * D + lane * E + e], o[e]);
      }
      bool bad = !(total_w * 0.f == 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) bad = bad || !(o[e] * 0.f == 0.f);
      const int t = P.by_group.over(T.row0 + r), h = kvh * P.group + T.row0 + r - t * P.group;
      const int64_t token = T.first + t;
      if (__any_sync(0xffffffffu, bad)) {
        const uint32_t w_lo = lo < T.W ? lo : T.W, w_hi = hi < T.W ? hi : T.W, f_lo = lo - w_lo, f_hi = hi - w_hi;   // of the window, behind it
        const uint32_t t_in = (uint32_t)(t - T.t_lo), nt = (uint32_t)T.nt;
        row_again<D>(P, b, (int)token, h, T.p_lo + (int)t_in, T.w0 + (int)w_lo, T.w0 + (int)w_hi, T.l - 1, T.dense,
                     T.m0 + (int)steps_below(f_lo, t_in, nt), T.m0 + (int)steps_below(f_hi, t_in, nt), o, mm, total_w);
      }
      if (active == 1) {
        finish<E>(P, token, h, lane, o, mm, total_w);
      } else {
        const int64_t at = ((int64_t)split * P.B.tokens + token) * P.heads + h;
#pragma unroll
        for (int e = 0; e < E; ++e) P.part_o[at * D + lane * E + e] = o[e];
        if (lane == 0) {
          P.part_m[at * 2] = mm;
          P.part_m[at * 2 + 1] = total_w;
        }
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------- ranges that meet
// a warp a row: the ranges' sums against the largest of their references.  How many ranges a row's list has is worked out as the first launch did
template <int D, bool TILES>
__global__ void __launch_bounds__(128) paged_join_kernel(const __grid_constant__ Params P, int tile_rows) {
  constexpr int E = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const int64_t row = (int64_t)blockIdx.x * 4 + warp, token = row / P.heads;
  if (token >= P.B.tokens) return;
  const int h = (int)(row - token * P.heads), b = sequence_of(P.B, (int)token, lane, &g_bad_rows);
  if (b < 0) return;
  const int64_t pair = (token - P.B.first[b]) * P.group + h % P.group;
  List T;
  if (!locate(T, P, b, (int)(pair / tile_rows), tile_rows)) return;
  int active;
  if (TILES) {
    int n0, n1, m0, m1;
    TileWalk(T, (int64_t)P.B.table_stride * P.C.page_size).range(P.splits, P.least, 0, n0, n1, m0, m1, active);
  } else {
    uint32_t lo, hi;
    T.range(P.splits, P.by_least, 0, lo, hi, active);
  }
  if (active == 1) return;
  // lane s: ranges s and s + 32 (there are 64 at most)
  const int64_t step = (int64_t)P.B.tokens * P.heads, at = token * P.heads + h;
  float2 stat[2] = {make_float2(-INFINITY, 0.f), make_float2(-INFINITY, 0.f)};
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (lane + 32 * u < active) stat[u] = *reinterpret_cast<const float2*>(P.part_m + (at + (lane + 32 * u) * step) * 2);
  float mm = fmaxf(stat[0].x, stat[1].x);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
  const float c0 = ex2(stat[0].x - reference(mm)), c1 = ex2(stat[1].x - reference(mm));
  const float sum = warp_sum(fmaf(c0, stat[0].y, c1 * stat[1].y));
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int s0 = 0; s0 < active; s0 += 8) {
    float v[8][E];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[u][e] = 0.f;
      if (s0 + u < active) {
        const float2* from = reinterpret_cast<const float2*>(P.part_o + (at + (s0 + u) * step) * D + lane * E);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 x = from[e / 2];
          v[u][e] = x.x;
          v[u][e + 1] = x.y;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float c = __shfl_sync(0xffffffffu, s0 + u < 32 ? c0 : c1, (s0 + u) & 31);
      if (s0 + u < active)
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(c, v[u][e], o[e]);
    }
  }
  finish<E>(P, token, h, lane, o, mm, sum);
}

// ---------------------------------------------------------------------------------------------- the call
// Which form, by what the few-row form would go through: entries of its lists, over all 16-row tiles.  Up to 16 rows it always serves (12 heads, 3000
// positions, 16 new tokens of 32 sequences 70 us, in 128-row tiles 86); beyond, a list that fills eight such tiles is better walked once.  Measured with 24 to
// 96 new tokens of 1, 8 and 32 sequences over 3000 positions, 12 heads, few rows / tiles in us: every position attended 14 / 23 (72 thousand entries),
// 22 / 24 (216), 39 / 29 (576), 45 / 31 (864), 88 / 86 (2304); stride 256, where tiles form a strided key for each row, 13 / 22 (86), 25 / 34 (258),
// 50 / 67 (516), 94 / 81 (1032); 4 x 512 tokens over 8192, stride 1024 89 / 43 (1790), stride 256 94 / 86 (1200), 4 x 2048 tokens 329 / 223.
// (A few-row form of 32 rows lost to the one of 16 in all of them.)
// The count of entries is not all: where strides are short against the lists, tiles form far more strided keys than they have tiles to cut a list by
// (TileWalk::range), and the rule takes them all the same.  Stride 64: 4 x 512 over 8192 222 / 306, 12 heads, 1024 tokens over 32768 429 / 606, and with 4
// heads, 512 tokens 98 / 560; stride 128, 20 heads on 4, 2 x 1024 over 16384 135 / 254; 128 columns, stride 256, 4 x 512 over 8192 129 / 163, 32 x 96 over 3000
// 117 / 122; strides below 64, whose masks tiles work out key by key, 4 x 512 over 2048 to 8192 stride 32 273 / 1091, stride 2 848 / 1102.
constexpr int TILE_ROWS = 128, FEW_ROWS = 16;
constexpr double TILES_FROM = 250e3, TILES_FROM_STRIDED = 900e3;
constexpr int64_t MOST_STEPS = 1 << 18;
constexpr int MOST_PAGES = 1 << 27;
Plan plan_of(const mst_paged_cache_t& c, const mst_paged_batch_t& b, int heads, int stride) {
  Plan p;
  const int group = heads / c.kv_heads;
  const int64_t new_tokens = b.max_new > 0 ? b.max_new : 1, rows = new_tokens * group, len = b.max_len > 0 ? b.max_len : 1;
  const int64_t lists = (int64_t)(b.batch > 0 ? b.batch : 1) * c.kv_heads;
  // entries of the longest list of a tile of `r` rows
  auto entries = [&](int r) {
    const int64_t in_tile = (r + group - 1) / group, nt = new_tokens < in_tile ? new_tokens : in_tile;
    return stride >= len || nt >= stride ? len : (stride + nt < len ? stride + nt : len) + len / stride * nt;
  };
  const bool strided = len / 2 >= stride && stride >= DENSE_BELOW;
  // What a tile does ahead of its first products some of its warps wait for, 0.8 s at least and not for ever: 2^18 strided keys take 0.4, to look through 2^27
  // pages for those that do not exist, 256 at a time, as long
  const int64_t reach = (int64_t)b.table_stride * c.page_size;
  p.tiles = rows > FEW_ROWS && group <= TILE_ROWS && b.table_stride < MOST_PAGES && (stride < DENSE_BELOW || reach / stride < MOST_STEPS) &&
            (double)lists * (double)((rows + FEW_ROWS - 1) / FEW_ROWS) * (double)entries(FEW_ROWS) >= (strided ? TILES_FROM_STRIDED : TILES_FROM);
  p.rows = p.tiles ? TILE_ROWS / group * group : rows <= FEW_ROWS / 2 ? FEW_ROWS / 2 : FEW_ROWS;
  const int64_t tiles = (rows + p.rows - 1) / p.rows;
  p.count = (int)(tiles < 65535 ? tiles : 65535);
  // Long lists are cut into ranges until there are blocks for the whole GPU, two of which an SM holds.  Tiles: no more than one wave (432 blocks of up to
  // 94 tiles: cut into 960 9 us more, when it took 272); at 128 columns, where an SM holds one block, that is two waves, which pays for lists of several lengths (300
  // to 900 new tokens over 2000 to 16000 positions, 8 heads, 99 us, for one wave 181; 1024 over 16384, 12 heads, 140 and 173) and costs where they are alike (1536
  // over 16384, 12 heads, 193 and 169; 128 over 32768, 8 heads, 54 and 42).  Few rows: for two, as lists are of many lengths (long ragged contexts 41.8 us, for six waves 47.9).
  // units: tiles of 128 keys and strided keys, which take about as long; or 64 entries
  int64_t units, want = 2 * (int64_t)mst_sm_count();
  if (p.tiles) {
    const int64_t nt = TILE_ROWS / group;
    units = (stride < DENSE_BELOW || stride + nt > len ? len : stride + nt) / KEYS_OF_TILE + 1 + (strided ? len / stride : 0);
  } else {
    units = (entries(p.rows) + UNIT - 1) / UNIT;
    want *= 2;
  }
  p.least = 8;      // 512 entries: a second launch costs as long as they take
  const int64_t blocks = lists * tiles, fit = (units + p.least - 1) / p.least;
  int64_t splits = p.tiles ? want / blocks : (want + blocks - 1) / blocks;
  if (splits > fit) splits = fit;
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  const int64_t each = (units + splits - 1) / splits;
  if (each > p.least) p.least = (int)(each < 0x7FFFFFFF ? each : 0x7FFFFFFF);
  p.splits = (int)splits;
  return p;
}
size_t workspace_of(const mst_paged_cache_t& c, const mst_paged_batch_t& b, int heads, const Plan& p) {
  if (p.splits <= 1) return 0;
  return (size_t)p.splits * (size_t)b.tokens * (size_t)heads * (size_t)(c.head_dim + 2) * sizeof(float);
}

template <int D, int NT>
mst_status_t launch_rows(const Params& P, const Plan& plan, cudaStream_t s) {
  const size_t smem = RowsShape<D>::SMEM;
  MST_SMEM_LIMIT((paged_rows_kernel<D, NT>), smem);
  const dim3 grid((unsigned)(plan.splits * P.C.kv_heads), (unsigned)plan.count, (unsigned)P.B.batch);
  MST_CUDA_TRY(mst_launch_overlapped(paged_rows_kernel<D, NT>, grid, dim3(32 * RW), smem, s, P));
  return MST_OK;
}
template <int D>
mst_status_t launch_rows(const Params& P, const Plan& plan, cudaStream_t s) {
  return plan.rows == FEW_ROWS / 2 ? launch_rows<D, 1>(P, plan, s) : launch_rows<D, 2>(P, plan, s);
}
template <int D>
mst_status_t launch_join(const Params& P, const Plan& plan, cudaStream_t s) {
  const unsigned blocks = (unsigned)(((int64_t)P.B.tokens * P.heads + 3) / 4);
  MST_CUDA_TRY(plan.tiles ? mst_launch_overlapped(paged_join_kernel<D, true>, dim3(blocks), dim3(128), 0, s, P, plan.rows)
                          : mst_launch_overlapped(paged_join_kernel<D, false>, dim3(blocks), dim3(128), 0, s, P, plan.rows));
  return MST_OK;
}

mst_status_t check_attention(const mst_paged_cache_t* cache, const mst_paged_batch_t* batch, int32_t heads, int32_t stride, Cache* C, Batch* B) {
  MST_TRY(check(cache, batch, C, B));
  if (heads <= 0 || stride <= 0) return MST_ERR_INVALID_ARG;
  if (heads % cache->kv_heads != 0 || heads > 65535) return MST_ERR_SHAPE;
  if (cache->head_dim != 64 && cache->head_dim != 128) return MST_ERR_SHAPE;
  // places in the cache are 32-bit numbers of 16-byte pieces
  if (((int64_t)cache->num_pages - 1) * (cache->page_stride / 8) + ((int64_t)cache->page_size - 1) * (cache->token_stride / 8) +
          ((int64_t)cache->kv_heads - 1) * (cache->head_stride / 8) + cache->head_dim / 8 >= 0xFFFFFFFFLL)
    return MST_ERR_SHAPE;
  return MST_OK;
}

}  // namespace

mst_status_t mst_paged_error_flags(int32_t* flags) {
  int32_t pages = 0, rows = 0, tiles = 0;
  MST_TRY(mst_paged::take_flag((const void*)&mst_paged::g_bad_page, &pages));
  MST_TRY(mst_paged::take_flag((const void*)&mst_paged::g_bad_rows, &rows));
  MST_TRY(mst_paged_tiles_error_flags(&tiles));
  *flags = pages | (rows << 2) | tiles;
  return MST_OK;
}

extern "C" mst_status_t mst_paged_attention_workspace(const mst_paged_cache_t* cache, const mst_paged_batch_t* batch, int32_t heads,
                                                      int32_t stride, size_t* bytes) {
  if (!bytes) return MST_ERR_INVALID_ARG;
  *bytes = 0;
  Cache C;
  Batch B;
  MST_TRY(check_attention(cache, batch, heads, stride, &C, &B));
  if (stride == 1) stride = 0x7FFFFFFF;
  *bytes = workspace_of(*cache, *batch, heads, plan_of(*cache, *batch, heads, stride));
  return MST_OK;
}

extern "C" mst_status_t mst_paged_attention(const mst_paged_cache_t* cache, const mst_paged_batch_t* batch, int32_t heads, int32_t stride,
                                            const void* Q, int64_t ldq, void* Out, int64_t ldo, float* lse, void* workspace,
                                            size_t workspace_bytes, mst_stream_t stream) {
  Params P = {};
  MST_TRY(check_attention(cache, batch, heads, stride, &P.C, &P.B));
  if (batch->tokens > 0 && (!Q || !Out)) return MST_ERR_INVALID_ARG;
  const int64_t width = (int64_t)heads * cache->head_dim;
  if (ldq < width || ldo < width || ldq % 8 != 0 || ldo % 8 != 0) return MST_ERR_SHAPE;
  if (((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(Out) | reinterpret_cast<uintptr_t>(workspace)) & 15u) != 0 ||
      (reinterpret_cast<uintptr_t>(lse) & 3u) != 0)
    return MST_ERR_SHAPE;
  if (stride == 1) stride = 0x7FFFFFFF;          // every distance is a multiple of one
  const Plan plan = plan_of(*cache, *batch, heads, stride);
  const size_t need = workspace_of(*cache, *batch, heads, plan);
  if (need > 0 && (!workspace || workspace_bytes < need)) return MST_ERR_CAPACITY;
  if (batch->batch == 0 || batch->tokens == 0) return MST_OK;
  if (need > 0 && ((int64_t)batch->tokens * heads + 3) / 4 > 0x7FFFFFFF) return MST_ERR_SHAPE;
  MST_TRY(mst_on_this_device({Q, Out, lse, need ? workspace : nullptr, P.C.K, P.C.V, P.B.first, P.B.len, P.B.table}));
  P.Q = (const __nv_bfloat16*)Q;
  P.Out = (__nv_bfloat16*)Out;
  P.lse = lse;
  P.ldq = ldq;
  P.ldo = ldo;
  P.heads = heads;
  P.group = heads / cache->kv_heads;
  P.by_group = Divider::of((uint32_t)P.group);
  P.l = stride;
  P.scale_log2 = LOG2E / sqrtf((float)cache->head_dim);
  P.splits = plan.splits;
  P.least = plan.least;
  P.by_l = Divider::of((uint32_t)stride);
  P.by_least = Divider::of((uint32_t)plan.least);
  P.part_o = (float*)workspace;
  if (need) P.part_m = P.part_o + (size_t)plan.splits * (size_t)batch->tokens * (size_t)heads * (size_t)cache->head_dim;
  cudaStream_t s = (cudaStream_t)stream;
  if (plan.tiles) MST_TRY(launch_tiles(P, plan, s));
  else MST_TRY(cache->head_dim == 64 ? launch_rows<64>(P, plan, s) : launch_rows<128>(P, plan, s));
  if (plan.splits > 1) MST_TRY(cache->head_dim == 64 ? launch_join<64>(P, plan, s) : launch_join<128>(P, plan, s));
  return MST_OK;
}
