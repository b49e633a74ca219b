// Attention of new tokens over a paged cache, the serving form of the strided attention:
//   Out = sum_{j in S_i} softmax_j(q . k_j / sqrt(d)) v_j,   S_i = { j <= i : i - j < l  or  (i - j) mod l == 0 }.
// Tiles of rows and the lists of keys they look at: mst_paged_list.h.  Few rows (one token, drafts): paged_rows_kernel, a block per (tile, key head,
// sequence, range of the list).
#include <cuda_bf16.h>

#include "mst_attention_tile.cuh"
#include "mst_internal.cuh"
#include "mst_paged.cuh"

namespace {
using namespace mst_ptx;
using mst_att::ex2;
using mst_att::ldsm_x4;
using mst_att::ldsm_x4_t;
using mst_att::mma_bf16;
using mst_paged::Batch;
using mst_paged::Cache;
using mst_paged::Key;
using mst_paged::List;

__device__ int g_bad_page = 0;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LAZY = 16.f;     // the reference of a softmax follows the maximum once that has moved up by 2^16: fp32 sums and bf16 weights lose nothing by it

struct Params {
  Cache C;
  Batch B;
  const __nv_bfloat16* Q;
  __nv_bfloat16* Out;
  float* lse;
  int64_t ldq, ldo;
  int heads, group, l;
  float scale_log2;
  int splits, least;      // most ranges of a list, and the least units of one (plan)
  float* part_o;          // [splits][tokens * heads][D]: sums against part_m, [splits][tokens * heads][2]: reference and sum of weights
  float* part_m;
};

constexpr int UNIT = 64;  // keys of a list that stay together

// A tile of sequence b (mst_paged_list.h)
__device__ __forceinline__ bool locate(List& T, const Params& P, int b, int tile, int R) {
  const int len = P.B.len[b];
  const int64_t reach = (int64_t)P.B.table_stride * P.C.page_size;
  if (!T.locate(P.B.first[b], P.B.first[b + 1], len, P.B.tokens, P.group, P.l, reach, tile, R)) return false;
  if (len > reach) g_bad_page = 1;
  return true;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// A row's sums -> its result, by one warp (lane: E neighbouring columns).  Nothing looked at: zeros and -inf
template <int E>
__device__ __forceinline__ void finish(const Params& P, int64_t token, int h, int lane, const float (&o)[E], float m, float sum) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint32_t w[E / 2];
#pragma unroll
  for (int e = 0; e < E / 2; ++e) w[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
  uint32_t* out = reinterpret_cast<uint32_t*>(P.Out + token * P.ldo + (int64_t)h * (32 * E)) + lane * (E / 2);
#pragma unroll
  for (int e = 0; e < E / 2; ++e) out[e] = w[e];
  if (P.lse && lane == 0) P.lse[(int64_t)h * P.B.tokens + token] = (m + log2f(sum)) * LN2;
}

// A row whose sums are not finite, formed again by one warp over the entries it looks at alone: what the matrix products multiplied by a weight
// of zero may have been infinite or NaN.  Lane: D / 32 neighbouring columns.
template <int D>
__device__ __noinline__ void row_again(const Params& P, const List T, int b, int kvh, int row, uint32_t lo, uint32_t hi, float (&o)[D / 32], float& m,
                                       float& sum) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int t = (T.row0 + row) / P.group, h = kvh * P.group + (T.row0 + row) % P.group;
  const __nv_bfloat16* q = P.Q + (int64_t)(T.first + t) * P.ldq + (int64_t)h * D + lane * E;
  m = -INFINITY;
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (uint32_t n = lo; n < hi; ++n) {
    const Key k = T.key(n);
    if (!T.sees(T.p_lo + t - T.t_lo, t - T.t_lo, k)) continue;
    const mst_paged::Slot s = mst_paged::slot_of(P.C, P.B, b, k.pos, &g_bad_page);
    if (!s.exists) continue;
    const int64_t at = s.at + (int64_t)kvh * P.C.head_stride + lane * E;
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) x = fmaf(__bfloat162float(q[e]), __bfloat162float(P.C.K[at + e]), x);
    x = warp_sum(x) * P.scale_log2;
    const float up = fmaxf(m, x);        // NaN: the weight below is NaN all the same
    const float c = ex2(m - reference(up)), w = ex2(x - reference(up));
    m = up;
    sum = fmaf(sum, c, w);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], c, w * __bfloat162float(P.C.V[at + e]));
  }
}

// ---------------------------------------------------------------------------------------------- few rows
// Four warps go through a range of the list, each through every fourth step of it with a ring of its own (no block-wide step until the
// end): K and V rows of a step come in by 16-byte asynchronous copies, two steps ahead; scores and weighted sums by warp-level products
// with the tile's rows in a 16-row operand, which costs less than the rows' bytes take to arrive however few of the 16 there are.  The
// warps' softmaxes are joined through shared memory, ranges by a second launch.
constexpr int RW = 4;             // warps
constexpr int RING = 3;
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

template <int D, int MT>
__global__ void __launch_bounds__(32 * RW) paged_rows_kernel(const __grid_constant__ Params P) {
  constexpr int R = 16 * MT, KEYS = RowsShape<D>::KEYS, STEP = RowsShape<D>::STEP_BYTES, PIECES = D / 8, AT_ONCE = 32 / PIECES;
  extern __shared__ unsigned char smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const int split = blockIdx.x, b = blockIdx.z;
  const int kvh = blockIdx.y % P.C.kv_heads;
  const uint32_t ring = ((smem_u32(smem_raw) + 127u) & ~127u) + (uint32_t)(warp * RowsShape<D>::WARP_BYTES);
  float* join = reinterpret_cast<float*>(smem_raw + (((smem_u32(smem_raw) + 127u) & ~127u) - smem_u32(smem_raw)));
  __shared__ float stat[RW][R][2];
  for (int tile = blockIdx.y / P.C.kv_heads;; tile += gridDim.y / P.C.kv_heads) {
    List T;
    if (!locate(T, P, b, tile, R)) return;
    uint32_t lo, hi;
    int active;
    if (!T.range(P.splits, P.least, UNIT, split, lo, hi, active)) continue;
    // queries: the 16 x 16 operand's published layout (row lane / 4 and + 8, columns 2 (lane % 4) and + 8)
    uint32_t q[MT][D / 16][4];
    int pos[MT][2], tok[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = mt * 16 + u * 8 + lane / 4, rr = r < T.rows ? r : 0;
        const int t = (T.row0 + rr) / P.group, h = kvh * P.group + (T.row0 + rr) % P.group;
        tok[mt][u] = t - T.t_lo;
        pos[mt][u] = T.p_lo + tok[mt][u];
        const uint32_t* src = reinterpret_cast<const uint32_t*>(P.Q + (int64_t)(T.first + t) * P.ldq + (int64_t)h * D) + lane % 4;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          q[mt][k][u] = src[k * 8];
          q[mt][k][u + 2] = src[k * 8 + 4];
        }
      }
    float acc[MT][D / 8][4], m[MT][2], sum[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int n = 0; n < D / 8; ++n) acc[mt][n][0] = acc[mt][n][1] = acc[mt][n][2] = acc[mt][n][3] = 0.f;
      m[mt][0] = m[mt][1] = -INFINITY;
      sum[mt][0] = sum[mt][1] = 0.f;
    }
    // step s of this warp: entries lo + (s RW + warp) KEYS ..; where they are is looked up a step before their copies go out
    Key keys[RING], next = {-1, -1};
    int64_t next_at = 0;
    auto look = [&](uint32_t s) {
      const uint64_t n = (uint64_t)lo + ((uint64_t)s * RW + warp) * KEYS + (KEYS == 32 ? lane : lane % 16);
      next = n < hi ? T.key((uint32_t)n) : Key{-1, -1};
      next_at = 0;
      if (next.pos >= 0) {
        const mst_paged::Slot sl = mst_paged::slot_of(P.C, P.B, b, next.pos, &g_bad_page);
        if (sl.exists) next_at = sl.at + (int64_t)kvh * P.C.head_stride;
        else next.pos = -1;
      }
    };
    auto load = [&](int slot) {
      keys[slot] = next;
      const uint32_t kt = ring + (uint32_t)(slot * 2 * STEP), vt = kt + STEP;
#pragma unroll
      for (int r0 = 0; r0 < KEYS; r0 += AT_ONCE) {
        const int r = r0 + lane / PIECES, c = lane % PIECES;
        const int64_t a = __shfl_sync(0xffffffffu, next_at, r);
        const bool there = __shfl_sync(0xffffffffu, next.pos, r) >= 0;
        cp16(piece<D>(kt, r, c), P.C.K + a + c * 8, there);
        cp16(piece<D>(vt, r, c), P.C.V + a + c * 8, there);
      }
    };
    const uint32_t total = (hi - lo + KEYS - 1) / KEYS;                                // steps of the block
    const uint32_t mine = total > (uint32_t)warp ? (total - warp + RW - 1) / RW : 0u;
#pragma unroll
    for (int s = 0; s < RING - 1; ++s) {
      look((uint32_t)s);
      if ((uint32_t)s < mine) load(s);
      cp_commit();
    }
    look(RING - 1);
    for (uint32_t s0 = 0; s0 < mine; s0 += RING) {
#pragma unroll
      for (int slot = 0; slot < RING; ++slot) {
        const uint32_t s = s0 + slot;
        if (s >= mine) break;
        cp_wait<RING - 2>();
        __syncwarp();                      // every lane's copies are in, and the slot to be filled has been read by every lane
        if (s + RING - 1 < mine) {
          load((slot + RING - 1) % RING);
          look(s + RING);
        }
        cp_commit();
        const uint32_t kt = ring + (uint32_t)(slot * 2 * STEP), vt = kt + STEP;
        float x[MT][KEYS / 8][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int n = 0; n < KEYS / 8; ++n) x[mt][n][0] = x[mt][n][1] = x[mt][n][2] = x[mt][n][3] = 0.f;
#pragma unroll
        for (int n = 0; n < KEYS / 8; ++n)
#pragma unroll
          for (int k2 = 0; k2 < D / 32; ++k2) {
            uint32_t f[4];
            ldsm_x4(f, piece<D>(kt, n * 8 + (lane & 7), k2 * 4 + (lane >> 3)));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              mma_bf16(x[mt][n], q[mt][2 * k2], f[0], f[1]);
              mma_bf16(x[mt][n], q[mt][2 * k2 + 1], f[2], f[3]);
            }
          }
        const Key key = keys[slot];
        const bool all = key.pos >= 0 && (key.who >= 0 ? T.nt == 1 : key.pos <= T.p_lo && T.p_hi - key.pos < T.l);
        if (!__all_sync(0xffffffffu, all)) {
#pragma unroll
          for (int n = 0; n < KEYS / 8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int from = n * 8 + 2 * (lane & 3) + e;
              const Key k = {__shfl_sync(0xffffffffu, key.pos, from), __shfl_sync(0xffffffffu, key.who, from)};
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                  if (!T.sees(pos[mt][u], tok[mt][u], k)) x[mt][n][2 * u + e] = -INFINITY;
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int n = 0; n < KEYS / 8; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) top[u] = fmaxf(top[u], fmaxf(x[mt][n][2 * u], x[mt][n][2 * u + 1]));
          top[0] *= P.scale_log2;
          top[1] *= P.scale_log2;
          if (__any_sync(0xffffffffu, top[0] > m[mt][0] + LAZY || top[1] > m[mt][1] + LAZY)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 1));
              top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 2));
              const bool up = top[u] > m[mt][u] + LAZY;
              const float c = up ? ex2(m[mt][u] - top[u]) : 1.f;
              if (up) m[mt][u] = top[u];
              sum[mt][u] *= c;
#pragma unroll
              for (int n = 0; n < D / 8; ++n) {
                acc[mt][n][2 * u] *= c;
                acc[mt][n][2 * u + 1] *= c;
              }
            }
          }
          const float r0 = reference(m[mt][0]), r1 = reference(m[mt][1]);
#pragma unroll
          for (int n = 0; n < KEYS / 8; ++n) {
            x[mt][n][0] = ex2(fmaf(x[mt][n][0], P.scale_log2, -r0));
            x[mt][n][1] = ex2(fmaf(x[mt][n][1], P.scale_log2, -r0));
            x[mt][n][2] = ex2(fmaf(x[mt][n][2], P.scale_log2, -r1));
            x[mt][n][3] = ex2(fmaf(x[mt][n][3], P.scale_log2, -r1));
            sum[mt][0] += x[mt][n][0] + x[mt][n][1];
            sum[mt][1] += x[mt][n][2] + x[mt][n][3];
          }
        }
#pragma unroll
        for (int k = 0; k < KEYS / 16; ++k) {
          uint32_t a[MT][4];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            a[mt][0] = pack_bf16(x[mt][2 * k][0], x[mt][2 * k][1]);
            a[mt][1] = pack_bf16(x[mt][2 * k][2], x[mt][2 * k][3]);
            a[mt][2] = pack_bf16(x[mt][2 * k + 1][0], x[mt][2 * k + 1][1]);
            a[mt][3] = pack_bf16(x[mt][2 * k + 1][2], x[mt][2 * k + 1][3]);
          }
#pragma unroll
          for (int n2 = 0; n2 < D / 16; ++n2) {
            uint32_t f[4];
            ldsm_x4_t(f, piece<D>(vt, k * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, n2 * 2 + (lane >> 4)));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              mma_bf16(acc[mt][2 * n2], a[mt], f[0], f[1]);
              mma_bf16(acc[mt][2 * n2 + 1], a[mt], f[2], f[3]);
            }
          }
        }
        __syncwarp();
      }
    }
    cp_wait<0>();
    // the warps' softmaxes meet in the rings' place
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = mt * 16 + u * 8 + lane / 4;
        float v = sum[mt][u];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        if ((lane & 3) == 0) {
          stat[warp][r][0] = m[mt][u];
          stat[warp][r][1] = v;
        }
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
          *reinterpret_cast<float2*>(join + ((warp * R + r) * D + n * 8 + 2 * (lane & 3))) = make_float2(acc[mt][n][2 * u], acc[mt][n][2 * u + 1]);
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
      if (__any_sync(0xffffffffu, bad)) row_again<D>(P, T, b, kvh, r, lo, hi, o, mm, total_w);
      const int t = (T.row0 + r) / P.group, h = kvh * P.group + (T.row0 + r) % P.group;
      const int64_t token = T.first + t;
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
// a warp a row: the ranges' sums against the largest of their references
template <int D, int R>
__global__ void __launch_bounds__(128) paged_join_kernel(const __grid_constant__ Params P) {
  constexpr int E = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const int b = blockIdx.z, kvh = blockIdx.y % P.C.kv_heads;
  for (int tile = blockIdx.y / P.C.kv_heads;; tile += gridDim.y / P.C.kv_heads) {
    List T;
    if (!locate(T, P, b, tile, R)) return;
    uint32_t lo, hi;
    int active;
    T.range(P.splits, P.least, UNIT, 0, lo, hi, active);
    if (active == 1) continue;
    for (int r = blockIdx.x * 4 + warp; r < T.rows; r += 4 * gridDim.x) {
      const int t = (T.row0 + r) / P.group, h = kvh * P.group + (T.row0 + r) % P.group;
      const int64_t token = T.first + t, step = (int64_t)P.B.tokens * P.heads, at = token * P.heads + h;
      float mm = -INFINITY;
      for (int s = 0; s < active; ++s) mm = fmaxf(mm, P.part_m[(at + s * step) * 2]);
      float sum = 0.f, o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
      for (int s = 0; s < active; ++s) {
        const float c = ex2(P.part_m[(at + s * step) * 2] - reference(mm));
        sum = fmaf(c, P.part_m[(at + s * step) * 2 + 1], sum);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(c, P.part_o[(at + s * step) * D + lane * E + e], o[e]);
      }
      finish<E>(P, token, h, lane, o, mm, sum);
    }
  }
}

// ---------------------------------------------------------------------------------------------- the call
struct Plan {
  int rows;           // of a tile
  int tiles, splits, least;
};
Plan plan_of(const mst_paged_cache_t& c, const mst_paged_batch_t& b, int heads, int stride) {
  Plan p;
  const int group = heads / c.kv_heads;
  const int64_t rows = (int64_t)(b.max_new > 0 ? b.max_new : 1) * group;
  p.rows = rows <= 16 ? 16 : 32;
  int64_t tiles = (rows + p.rows - 1) / p.rows;
  const int64_t most = 65535 / c.kv_heads;
  p.tiles = (int)(tiles < most ? tiles : most);
  // entries of the longest list
  const int64_t nt = (p.rows + group - 1) / group, len = b.max_len > 0 ? b.max_len : 1;
  const int64_t list = stride >= len || nt >= stride ? len : (stride + nt < len ? stride + nt : len) + len / stride * nt;
  const int64_t blocks = (int64_t)(b.batch > 0 ? b.batch : 1) * c.kv_heads * tiles, want = 12 * (int64_t)mst_sm_count();
  int64_t splits = (want + blocks - 1) / blocks;
  p.least = 4;
  const int64_t units = (list + UNIT - 1) / UNIT, fit = (units + p.least - 1) / p.least;
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

template <int D, int MT>
mst_status_t launch_rows(const Params& P, const Plan& plan, cudaStream_t s) {
  const size_t smem = RowsShape<D>::SMEM;
  MST_SMEM_LIMIT((paged_rows_kernel<D, MT>), smem);
  const unsigned y = (unsigned)(plan.tiles * P.C.kv_heads), z = (unsigned)P.B.batch;
  MST_CUDA_TRY(mst_launch_overlapped(paged_rows_kernel<D, MT>, dim3((unsigned)plan.splits, y, z), dim3(32 * RW), smem, s, P));
  if (plan.splits > 1) MST_CUDA_TRY(mst_launch_overlapped(paged_join_kernel<D, 16 * MT>, dim3(4 * MT, y, z), dim3(128), 0, s, P));
  return MST_OK;
}

mst_status_t check_attention(const mst_paged_cache_t* cache, const mst_paged_batch_t* batch, int32_t heads, int32_t stride, Cache* C, Batch* B) {
  MST_TRY(mst_paged::check(cache, batch, C, B));
  if (heads <= 0 || stride <= 0) return MST_ERR_INVALID_ARG;
  if (heads % cache->kv_heads != 0 || heads > 65535) return MST_ERR_SHAPE;
  if (cache->head_dim != 64 && cache->head_dim != 128) return MST_ERR_SHAPE;
  return MST_OK;
}

}  // namespace

mst_status_t mst_paged_error_flags(int32_t* flags) { return mst_paged::take_flag((const void*)&g_bad_page, flags); }

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
  if (!Q || !Out) return MST_ERR_INVALID_ARG;
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
  MST_TRY(mst_on_this_device({Q, Out, lse, need ? workspace : nullptr, P.C.K, P.C.V, P.B.first, P.B.len, P.B.table}));
  P.Q = (const __nv_bfloat16*)Q;
  P.Out = (__nv_bfloat16*)Out;
  P.lse = lse;
  P.ldq = ldq;
  P.ldo = ldo;
  P.heads = heads;
  P.group = heads / cache->kv_heads;
  P.l = stride;
  P.scale_log2 = LOG2E / sqrtf((float)cache->head_dim);
  P.splits = plan.splits;
  P.least = plan.least;
  P.part_o = (float*)workspace;
  if (need) P.part_m = P.part_o + (size_t)plan.splits * (size_t)batch->tokens * (size_t)heads * (size_t)cache->head_dim;
  cudaStream_t s = (cudaStream_t)stream;
  if (cache->head_dim == 64) return plan.rows == 16 ? launch_rows<64, 1>(P, plan, s) : launch_rows<64, 2>(P, plan, s);
  return plan.rows == 16 ? launch_rows<128, 1>(P, plan, s) : launch_rows<128, 2>(P, plan, s);
}
