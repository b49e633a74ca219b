// Attention over a paged cache for many rows (chunks of prompts): tiles of up to 128 (token, head) rows of one key head on the tensor cores.
// Keys come in tiles of 128 positions (mst_paged_list.h: TileWalk); the strided keys further back, which one row each looks at, are formed row by
// row and are where the first half's softmax starts.  Roles of a block's ten warps:
//   warps 0-7  softmax: thread = row (tensor-memory lane), the two warps of a lane quarter take 64 of a tile's 128 keys each.  The halves are
//              pipelines of their own - scores, weights, reference, sum, output accumulator - that share the loads only and meet when the rows
//              leave: one's products are under way while the other takes exponentials;
//   warp 8     fills rings of two key and two value tiles: pages whose positions fall on whole boxes by TMA, a box at most 64 rows high; the tile
//              in which a sequence ends, pages that do not exist and page sizes without a factor of eight by 16-byte asynchronous copies, zeros
//              where nothing is (what a page holds behind the length may be no number);
//   warp 9     tcgen05.mma: S_half = Q K_half^T (128 x 64), O_half += P_half V_half, P read from tensor memory where the softmax warps have
//              written it over the scores.
// Tensor memory: the halves' scores in columns 0-63 and 64-127, their outputs behind: two blocks an SM at head_dim 64.  Ranges of a list (blockIdx.x)
// leave sums for the join.
// Bound: the chain of a half through products, exponentials and barriers, four of which an SM has at a time: 2900 clocks for a 128 x 128 tile of each of
// the two blocks, of which the exponential unit (16 a clock) needs 2048 and the products 640.  4479 tokens of three sequences over 4000 to 12000
// positions, 12 heads: 185 us.  Taken back: tiles of 64 keys with two score buffers (33 us more), tiles of 128 without independent halves (32), one lane
// that issues by itself (5); an eighth of the exponentials as polynomials (6 us less, a quarter nothing: not worth a second exponential); blocks that
// take even shares of all tiles' keys (when tiles came sequence by sequence: 8 us less here, but 4 x 1024 tokens 26 -> 102, 32 x 512 of 600 82 -> 230:
// what a block does at its start and end is then done by few blocks one after another).
#include <cuda.h>

#include <type_traits>

#include "mst_paged_attention.cuh"

namespace {
using namespace mst_paged;
using namespace mst_att;
using mst_ptx::pack_bf16;

__device__ int g_wait_error = 0;

constexpr int STAGES = 2;
constexpr int KEYS = KEYS_OF_TILE;
template <int D_>
struct Shape {
  static constexpr int PARTS = D_ / 64;                            // 64 columns each: 128 bytes a row
  static constexpr int OWN_BYTES = PARTS * 2 * TILE_BYTES;
  static constexpr int SLOT_BYTES = PARTS * 2 * TILE_BYTES;        // 128 keys, or their values
  static constexpr int TMEM_COLS = D_ == 64 ? 256 : 512;
  static constexpr int BLOCKS = D_ == 64 ? 2 : 1;
  // own rows, rings, statistics, which keys exist, barriers (full and empty of both rings, own_full, s_full[2], p_full[2], acc_full, far_over)
  static constexpr int SMEM = OWN_BYTES + STAGES * 2 * SLOT_BYTES + 3 * 2 * ROWS * 4 + STAGES * 16 + 32 * STAGES + 7 * 8 + 1024;
};

struct TileParams {
  Params P;
  int rows;             // of a tile: whole tokens
  Divider by_tokens;    // how many, and one over that
  float per_token;
  int count;            // tiles of a sequence that the grid has
  int box;              // rows of a TMA box, 0: plain copies only
  int at_slot, at_head, at_page;   // which of the map's coordinates 1 .. 3 they are
};

__device__ __forceinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return mbar_wait(bar, parity, abort_flag, &g_wait_error);
}
constexpr float MOST = 65536.f;
__device__ __forceinline__ float halves_sum(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(tm),
               "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(tm), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one;
}
__device__ __forceinline__ void tmem_ld8_nowait(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_ld8_wait(uint32_t (&r)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
               :
               : "memory");
}
// The instructions of a whole warp of which the elected lane's counts: no branch around them, so that what they name stays uniform
__device__ __forceinline__ void mma_ss(uint32_t one, uint32_t d, uint64_t a, uint64_t b, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(IDESC_K), "r"(accum), "r"(one)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t one, uint32_t d, uint32_t a, uint64_t b, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(IDESC_MN), "r"(accum), "r"(one)
      : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t one, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(one)
      : "memory");
}
__device__ __forceinline__ void softmax_warps_meet() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------- strided keys of a row
// Two lanes a row, D / 2 columns each, from the caller's memory
template <int W>
struct Half {
  uint32_t w[W];      // W pairs of values
};
template <int W>
__device__ __forceinline__ void half_row(Half<W>& x, const __nv_bfloat16* p, bool there) {
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (there) v = *reinterpret_cast<const uint4*>(p + 2 * i);
    x.w[i] = v.x; x.w[i + 1] = v.y; x.w[i + 2] = v.z; x.w[i + 3] = v.w;
  }
}
template <int W>
__device__ __forceinline__ float half_dot(const Half<W>& a, const Half<W>& b) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < W; ++e) {
    uint16_t al, ah, bl, bh;
    halves(a.w[e], al, ah);
    halves(b.w[e], bl, bh);
    fma_bf16(s[e & 1], al, bl);
    fma_bf16(s[2 + (e & 1)], ah, bh);
  }
  const float x = (s[0] + s[1]) + (s[2] + s[3]);
  return x + __shfl_xor_sync(0xffffffffu, x, 16);
}
// the sums of sixteen rows -> tensor memory from lane rs on: lanes 0-15 of the warp hold columns 0 .. D / 2 - 1, lanes 16-31 the others
__device__ __forceinline__ void start_sums(uint32_t taddr, const float (&a)[32]) { far_start_sums(taddr, a); }
__device__ __forceinline__ void start_sums(uint32_t taddr, const float (&a)[64]) {
#pragma unroll
  for (int g = 0; g < 2; ++g)
    asm volatile(
        "tcgen05.st.sync.aligned.16x32bx2.x32.b32 [%32], 64, "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"f"(a[32 * g + 0]),
        "f"(a[32 * g + 1]), "f"(a[32 * g + 2]), "f"(a[32 * g + 3]), "f"(a[32 * g + 4]), "f"(a[32 * g + 5]), "f"(a[32 * g + 6]), "f"(a[32 * g + 7]),
        "f"(a[32 * g + 8]), "f"(a[32 * g + 9]), "f"(a[32 * g + 10]), "f"(a[32 * g + 11]), "f"(a[32 * g + 12]), "f"(a[32 * g + 13]),
        "f"(a[32 * g + 14]), "f"(a[32 * g + 15]), "f"(a[32 * g + 16]), "f"(a[32 * g + 17]), "f"(a[32 * g + 18]), "f"(a[32 * g + 19]),
        "f"(a[32 * g + 20]), "f"(a[32 * g + 21]), "f"(a[32 * g + 22]), "f"(a[32 * g + 23]), "f"(a[32 * g + 24]), "f"(a[32 * g + 25]),
        "f"(a[32 * g + 26]), "f"(a[32 * g + 27]), "f"(a[32 * g + 28]), "f"(a[32 * g + 29]), "f"(a[32 * g + 30]), "f"(a[32 * g + 31]),
        "r"(taddr + 32u * g)
        : "memory");
}

// What a call's lists can have: nothing behind the window (NEAR: no position is two strides in), strided keys row by row (FAR), or the set in the
// mask of every tile (DENSE: short strides).  Code that is only jumped over costs registers here.
enum Mode { NEAR, FAR, DENSE };

// Which tile of rows comes n-th.  Those with the most keys first, so that no long list starts late: a sequence's from its end, and over all sequences where
// there are 32 at most and they do not end alike.  A warp's question then, each lane with a sequence: tiles lie on levels of as many positions as a tile
// has tokens, a sequence's on successive ones, and the level that has the n-th is found by halving.  Where one launch has chunks of long and of short
// sequences: 4479 tokens of three over 4000 to 12000 positions 256 -> 185 us, 4 x 375 to 1500 over 1500 to 9000 164 -> 130, 16 x 512 to 2048 over 2048 to
// 4000 316 -> 297, stride 256 266 -> 237; where all end alike the question costs 1 to 3 % (16 x 1024 88.4 -> 90.7 us).
struct Turn {
  int b, tile, first, end, len;     // a sequence, its tile (-1: none), its rows and its length (RowsOf)
  static __device__ __forceinline__ int count(const TileParams& A, int first, int end) {      // of RowsOf
    return first >= 0 && end > first ? A.by_tokens.over(end - first - 1) + 1 : 0;
  }
  __device__ __forceinline__ Turn(const TileParams& A, uint32_t z, int lane) {
    const Batch& B = A.P.B;
    const bool few = B.batch <= 32;
    const int mine = few ? (lane < B.batch ? lane : 0) : (int)blockIdx.y;
    const RowsOf rows(B.first[mine], B.first[mine + 1], B.len[mine], B.tokens);
    if (rows.outside) g_bad_rows = 1;
    first = rows.first;
    end = rows.end;
    len = rows.len;
    b = (int)blockIdx.y;
    int tiles = count(A, first, end);
    tile = tiles - 1 - (int)z;
    if (!few) return;
    if (lane >= B.batch) tiles = 0;
    constexpr float FAR_OFF = 1 << 29;
    const float level = ((float)len - (float)(end - first)) * A.per_token;       // about: a sequence may be off by a little
    const int below = (int)fminf(fmaxf(level, -FAR_OFF), FAR_OFF), top = below + tiles;
    int hi = __reduce_max_sync(0xffffffffu, tiles > 0 ? top : -(1 << 30));
    if (hi - __reduce_min_sync(0xffffffffu, tiles > 0 ? top : 1 << 30) > 1) {
      auto from = [&](int level) {      // tiles on this level or above
        const int n = top - level + 1;
        return __reduce_add_sync(0xffffffffu, (uint32_t)(n < 0 ? 0 : n < tiles ? n : tiles));
      };
      const uint32_t n = blockIdx.y + z * (uint32_t)B.batch;
      int lo = __reduce_min_sync(0xffffffffu, tiles > 0 ? below + 1 : 1 << 30);
      while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (from(mid) > n) lo = mid;
        else hi = mid - 1;
      }
      uint32_t on = __ballot_sync(0xffffffffu, lo > below && lo <= top);
      for (uint32_t skip = n - from(lo + 1); skip > 0 && on; --skip) on &= on - 1;
      b = on ? __ffs(on) - 1 : 0;
      tile = on ? __reduce_max_sync(0xffffffffu, lane == b ? lo - 1 - below : -1) : -1;
    } else {
      tile = __shfl_sync(0xffffffffu, tile, b);
    }
    first = __shfl_sync(0xffffffffu, first, b);
    end = __shfl_sync(0xffffffffu, end, b);
    len = __shfl_sync(0xffffffffu, len, b);
  }
};

template <int D_, Mode MODE>
__global__ void __launch_bounds__(THREADS, Shape<D_>::BLOCKS)
paged_tiles_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                   const __grid_constant__ TileParams A) {
  using S = Shape<D_>;
  constexpr int PARTS = S::PARTS, HALF = D_ / 2, OUT0 = 128;     // OUT0: tensor-memory column of the first half's outputs
  const Params& P = A.P;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t own = (smem_u32(smem_raw) + 1023u) & ~1023u, ring_k = own + S::OWN_BYTES, ring_v = ring_k + STAGES * S::SLOT_BYTES,
                 stat_a = ring_v + STAGES * S::SLOT_BYTES;
  const uint32_t exist_a = stat_a + 3 * 2 * ROWS * 4, full_k = exist_a + 16 * STAGES, full_v = full_k + 8 * STAGES, empty_k = full_v + 8 * STAGES,
                 empty_v = empty_k + 8 * STAGES, own_full = empty_v + 8 * STAGES, s_full = own_full + 8, p_full = s_full + 16, acc_full = p_full + 16,
                 far_over = acc_full + 8;
  unsigned char* base = smem_raw + (own - smem_u32(smem_raw));
  volatile uint32_t* exist = reinterpret_cast<uint32_t*>(base + (exist_a - own));     // [STAGES][4]
  __shared__ uint32_t holder;
  __shared__ uint32_t again[ROWS / 32];
  __shared__ int abort_sh;
  volatile int* abort_flag = &abort_sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    abort_sh = 0;
    for (int s = 0; s < 4 * STAGES; ++s) mbar_init(full_k + 8 * s, 1);
    mbar_init(own_full, 1);
    for (int h = 0; h < 2; ++h) {
      mbar_init(s_full + 8 * h, 1);
      mbar_init(p_full + 8 * h, CW / 2);
    }
    mbar_init(acc_full, 1);
    mbar_init(far_over, CW);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x < ROWS / 32) again[threadIdx.x] = 0u;
  if (warp == CW && lane < 3) prefetch_map(lane == 0 ? &tmQ : lane == 1 ? &tmK : &tmV);
  if (warp == CW + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&holder)), "r"(S::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = holder;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();

  const int kvh = (int)blockIdx.x % P.C.kv_heads, split = (int)blockIdx.x / P.C.kv_heads;
  const int64_t reach = (int64_t)P.B.table_stride * P.C.page_size;
  uint32_t lap = 0, far_lap = 0;   // tiles of rows so far, those with strided keys: barriers that complete once in each
  uint32_t base_t = 0;  // near tiles so far: ring places go on from tile to tile
  for (uint32_t z = blockIdx.z;; z += (uint32_t)A.count) {
    const Turn turn_of(A, z, lane);
    const int b = turn_of.b, len = turn_of.len, have = (int)(len < reach ? len : reach);       // positions that there are
    List T;
    if (turn_of.tile < 0 || !T.locate(turn_of.first, turn_of.end, len, P.B.tokens, P.by_group, P.by_l, reach, turn_of.tile, A.rows)) break;
    if (len > reach) g_bad_page = 1;
    const TileWalk walk(T, reach);
    int n0, n1, m0, m1, active;
    if (!walk.range(P.splits, P.least, split, n0, n1, m0, m1, active)) continue;
    const int near = n1 - n0, key0 = walk.first + n0 * KEYS;
    if (near == 0) {      // no row has a position
      if (warp < CW)
        for (int r = warp; r < T.rows; r += CW) {
          const float none[D_ / 32] = {};
          finish<D_ / 32>(P, T.first + (T.row0 + r) / P.group, kvh * P.group + (T.row0 + r) % P.group, lane, none, -INFINITY, 0.f);
        }
      continue;
    }
    const int32_t* table = P.B.table + (int64_t)b * P.B.table_stride;
    // A wait that gives up sets the block's abort flag, after which every wait returns at once: nobody leaves his loop early, and nothing is stored
    if (warp == CW) {
      // ------------------------------------------------------------------------------------------ loads
      if (lane == 0) {
        mbar_expect_tx(own_full, (uint32_t)(A.rows * D_ * 2));
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
          tma_load_3d(own + c * 2 * TILE_BYTES, &tmQ, 64 * c, kvh * P.group, T.first + T.t_lo, own_full);
      }
      bool waiting = false;  // plain copies of the tile before are under way
      auto give = [&](uint32_t n) {
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(full_k + 8 * (n % STAGES));
          mbar_arrive(full_v + 8 * (n % STAGES));
        }
        waiting = false;
      };
      for (int j = 0; j < near; ++j) {
        const uint32_t n = base_t + (uint32_t)j, s = n % STAGES;
        const int k0 = key0 + j * KEYS;
        const uint32_t to_k = ring_k + s * S::SLOT_BYTES, to_v = ring_v + s * S::SLOT_BYTES;
        bool whole = A.box > 0 && KEYS <= have - k0;
        int id = 0, slot = 0;
        const bool mine = whole && lane * A.box < KEYS;
        if (mine) id = page_of(table, P.B.table_stride, P.C.by_page, P.C.num_pages, k0 + lane * A.box, slot);
        whole = whole && __all_sync(0xffffffffu, id >= 0);
        const uint32_t before = (n / STAGES - 1) & 1u;
        if (waiting) {        // ahead of any wait for a slot: the products of the tile before that one may be waiting for these keys
          cp_wait<0>();
          give(n - 1);
        }
        if (whole) {
          int c[4];
#pragma unroll
          for (int d = 1; d < 4; ++d) c[d] = d == A.at_slot ? slot : d == A.at_head ? kvh : id;
          if (n >= STAGES) wait_on(empty_k + 8 * s, before, abort_flag);
          __syncwarp();
          if (lane == 0) mbar_expect_tx(full_k + 8 * s, S::SLOT_BYTES);
          __syncwarp();
          if (mine)
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
              tma_load_4d(to_k + (uint32_t)(q * 2 * TILE_BYTES + lane * A.box * 128), &tmK, 64 * q, c[1], c[2], c[3], full_k + 8 * s);
          if (n >= STAGES) wait_on(empty_v + 8 * s, before, abort_flag);     // then nobody reads `exist` of the tile before either
          __syncwarp();
          if (lane < 4) exist[4 * s + lane] = ~0u;
          __syncwarp();
          if (lane == 0) mbar_expect_tx(full_v + 8 * s, S::SLOT_BYTES);
          __syncwarp();
          if (mine)
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
              tma_load_4d(to_v + (uint32_t)(q * 2 * TILE_BYTES + lane * A.box * 128), &tmV, 64 * q, c[1], c[2], c[3], full_v + 8 * s);
        } else {
          if (n >= STAGES) {
            wait_on(empty_k + 8 * s, before, abort_flag);
            wait_on(empty_v + 8 * s, before, abort_flag);
          }
          __syncwarp();
          constexpr int PIECES = D_ / 8, AT_ONCE = 32 / PIECES;
          const int c = lane % PIECES;
#pragma unroll 1
          for (int u = 0; u < KEYS / 32; ++u) {
            const int k = k0 + 32 * u + lane;
            int64_t at = 0;
            bool there = false;
            if (k < have) {
              const Slot sl = slot_of(P.C, P.B, b, k, &g_bad_page);
              there = sl.exists;
              if (sl.exists) at = sl.at + (int64_t)kvh * P.C.head_stride;
            }
            const uint32_t bits = __ballot_sync(0xffffffffu, there);
            if (lane == 0) exist[4 * s + u] = bits;
#pragma unroll 4
            for (int r0 = 0; r0 < 32; r0 += AT_ONCE) {
              const int r = r0 + lane / PIECES;
              const int64_t a = __shfl_sync(0xffffffffu, at, r);
              const bool in = (bits >> r) & 1u;
              const uint32_t to = piece_addr((uint32_t)(c / 8) * 2 * TILE_BYTES, 32 * u + r, c % 8);
              cp16(to_k + to, P.C.K + a + c * 8, in);
              cp16(to_v + to, P.C.V + a + c * 8, in);
            }
          }
          cp_commit();
          waiting = true;
        }
      }
      if (waiting) {
        cp_wait<0>();
        give(base_t + (uint32_t)near - 1);
      }
    } else if (warp == CW + 1) {
      // ------------------------------------------------------------------------------------------ products
      // The whole warp goes through the loop and one elected lane issues.  What the instructions name is the same in every turn, a slot's and a half's
      // part being constants, and there is no branch around them: a tile's sixteen products take 1000 clocks to issue (1300 in a branch of a lane).
      const uint32_t leader = elect_one();
      const uint64_t qd = smem_desc(own, 16, 1024), kd0 = smem_desc(ring_k, 16, 1024), vd0 = smem_desc(ring_v, 16, 1024);
      constexpr uint64_t step = S::SLOT_BYTES >> 4, part = (2 * TILE_BYTES) >> 4, half_tile = TILE_BYTES >> 4;
      const uint32_t from_far = MODE == FAR && m1 > m0 ? 1u : 0u;
      auto scores = [&](auto slot, auto half) {
        constexpr uint32_t SL = decltype(slot)::value, H = decltype(half)::value;
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            mma_ss(leader, tmem + H * 64u, qd + part * q + 2 * ks, kd0 + step * SL + part * q + half_tile * H + 2 * ks, (q > 0 || ks > 0) ? 1u : 0u);
        commit_to(leader, s_full + 8 * H);
        if (H == 1) commit_to(leader, empty_k + 8 * SL);
        __syncwarp();
      };
      auto outputs = [&](auto slot, auto half, uint32_t more, bool last) {
        constexpr uint32_t SL = decltype(slot)::value, H = decltype(half)::value;
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            mma_ts(leader, tmem + OUT0 + (uint32_t)(H * D_ + 64 * q), tmem + (uint32_t)(H * 64 + ks * 8),
                   vd0 + step * SL + part * q + half_tile * H + (uint64_t)(ks * ((16 * 128) >> 4)), ks ? 1u : more);
        if (H == 1) {
          commit_to(leader, empty_v + 8 * SL);
          if (last) commit_to(leader, acc_full);
        }
        __syncwarp();
      };
      constexpr std::integral_constant<uint32_t, 0> C0{};
      constexpr std::integral_constant<uint32_t, 1> C1{};
      // tile j in slot `here`: its weights are used up half by half, the next tile's scores follow in the other slot
      auto turn = [&](int j, auto here, auto there) {
        const uint32_t n = base_t + (uint32_t)j;
        const bool last = j + 1 == near;
        wait_on(full_v + 8 * (n % STAGES), (n / STAGES) & 1u, abort_flag);     // ahead of the weights: nothing but products between those and the scores
        if (!last) wait_on(full_k + 8 * ((n + 1) % STAGES), ((n + 1) / STAGES) & 1u, abort_flag);
        wait_on(p_full, n & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        outputs(here, C0, (j > 0 ? 1u : 0u) | from_far, last);
        if (!last) scores(there, C0);
        wait_on(p_full + 8, n & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        outputs(here, C1, j > 0 ? 1u : 0u, last);
        if (!last) scores(there, C1);
      };
      static_assert(STAGES == 2, "slots take turns");
      wait_on(own_full, lap & 1u, abort_flag);
      wait_on(full_k + 8 * (base_t % STAGES), (base_t / STAGES) & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
      if (base_t % 2 == 0) {
        scores(C0, C0);
        scores(C0, C1);
      } else {
        scores(C1, C0);
        scores(C1, C1);
      }
      for (int j = 0; j < near; ++j) {
        if ((base_t + (uint32_t)j) % 2 == 0) turn(j, C0, C1);
        else turn(j, C1, C0);
      }
    } else {
      // ------------------------------------------------------------------------------------------ softmax
      const int quarter = warp & 3, half = warp >> 2;
      const int r = quarter * 32 + lane, rs = quarter * 32 + half * 16;   // this thread's row; this warp's sixteen of the strided keys
      const uint32_t t_row = tmem + ((uint32_t)(quarter * 32) << 16), t_out = t_row + OUT0 + (uint32_t)half * D_;
      const uint64_t scale2 = pack2(P.scale_log2, P.scale_log2);
      float* stat = reinterpret_cast<float*>(base + (stat_a - own));      // [3][2][128]
      const bool live = r < T.rows;
      const int pos = live ? T.p_lo + (T.row0 + r) / P.group - T.t_lo : -1;
      const int w0 = quarter * 32, w1 = w0 + 31 < T.rows ? w0 + 31 : T.rows - 1;     // this warp's rows
      const int i_lo = T.p_lo + (T.row0 + w0) / P.group - T.t_lo, i_hi = w0 < T.rows ? T.p_lo + (T.row0 + w1) / P.group - T.t_lo : -1;
      // do all the range's pages exist (keys behind a sequence's end are behind every row of it)
      bool hole = len > reach;
      {
        const int64_t stop = (int64_t)key0 + (int64_t)near * KEYS;
        const int p1 = have > 0 ? P.C.by_page.over((int)(stop < have ? stop : have) - 1) : -1;
        for (int p = P.C.by_page.over(key0) + (int)threadIdx.x; p <= p1; p += 32 * CW) {
          const int id = table[p];
          hole = hole || id < 0 || id >= P.C.num_pages;
        }
        uint32_t any_hole;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 2, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
            : "=r"(any_hole)
            : "r"((uint32_t)hole)
            : "memory");
        hole = any_hole != 0u;
      }
      float m = -INFINITY;                                   // reference of this half's softmax, base 2
      float total_w = 0.f;
      if (MODE == FAR && m1 > m0) {
        const int fr = rs + (lane & 15);
        const bool there = fr < T.rows;
        const int fp = there ? T.p_lo + (T.row0 + fr) / P.group - T.t_lo : -1;
        const int col = (lane >> 4) * HALF;
        Half<HALF / 2> mine;
        half_row(mine, P.Q + (int64_t)(T.first + (there ? (T.row0 + fr) / P.group : 0)) * P.ldq + (int64_t)(kvh * P.group + (there ? (T.row0 + fr) % P.group : 0)) * D_ + col, there);
        float acc[HALF], fm = -INFINITY, fs = 0.f;
#pragma unroll
        for (int e = 0; e < HALF; ++e) acc[e] = 0.f;
        // A step's page is asked for a step ahead, its slot's place in the cache is worked out when the number is there
        struct Far { int id, slot; };
        auto look = [&](int k) {
          const int64_t j = (int64_t)fp - (int64_t)k * P.l;
          Far f = {-2, 0};                              // -2: before the sequence
          if (j >= 0 && k < m1) {
            const int page = P.C.by_page.over((int)j);
            f.slot = (int)j - page * P.C.page_size;
            f.id = page < P.B.table_stride ? __ldg(table + page) : -1;
          }
          return f;
        };
        Far next = look(m0);
        for (int k = m0; k < m1; ++k) {
          const Far now = next;
          next = look(k + 1);
          const bool exists = now.id >= 0 && now.id < P.C.num_pages;
          if (now.id != -2 && !exists) g_bad_page = 1;
          const int64_t at = exists ? (int64_t)now.id * P.C.page_stride + (int64_t)now.slot * P.C.token_stride + (int64_t)kvh * P.C.head_stride + col : 0;
          Half<HALF / 2> kk, vv;
          half_row(kk, P.C.K + at, exists);
          half_row(vv, P.C.V + at, exists);
          const float d = half_dot(mine, kk);          // every lane: it has a shuffle
          const float x = exists ? d * P.scale_log2 : -INFINITY;
          const bool up = x > fm + LAZY;
          if (__any_sync(0xffffffffu, up)) {
            const float c = up ? ex2(fm - x) : 1.f;
            if (up) fm = x;
            fs *= c;
#pragma unroll
            for (int e = 0; e < HALF; ++e) acc[e] *= c;
          }
          const float w = exists ? ex2(x - mst_paged::reference(fm)) : 0.f;
          fs += w;
          uint16_t wb, dummy;
          halves(pack_bf16(w, 0.f), wb, dummy);
#pragma unroll
          for (int e = 0; e < HALF / 2; ++e) {
            uint16_t lo, hi;
            halves(vv.w[e], lo, hi);
            fma_bf16(acc[2 * e], wb, lo);
            fma_bf16(acc[2 * e + 1], wb, hi);
          }
        }
        start_sums(tmem + ((uint32_t)rs << 16) + OUT0, acc);
        if (lane < 16) {
          stat[4 * ROWS + rs + lane] = fm;
          stat[5 * ROWS + rs + lane] = fs;
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(far_over);
        wait_on(far_over, far_lap & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        if (half == 0) {
          m = stat[4 * ROWS + r];
          total_w = stat[5 * ROWS + r];
        }
      }
      for (int j = 0; j < near; ++j) {
        const uint32_t n = base_t + (uint32_t)j;
        if (hole) wait_on(full_v + 8 * (n % STAGES), (n / STAGES) & 1u, abort_flag);       // with it `exist`
        wait_on(s_full + 8 * half, n & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
        const int k0 = key0 + j * KEYS + half * 64;            // this warp's keys: k0 .. k0 + 63
        uint32_t there[2] = {~0u, ~0u};
        if (hole) {
          there[0] = exist[4 * (n % STAGES) + 2 * half];
          there[1] = exist[4 * (n % STAGES) + 2 * half + 1];
        }
        const uint32_t t_s = t_row + (uint32_t)(half * 64);
        uint32_t w[32];
        if ((there[0] | there[1]) && i_hi >= k0 && (MODE == DENSE || i_lo - (k0 + 63) <= P.l)) {      // some pair may be attended
          const bool some_not = MODE == DENSE || (there[0] & there[1]) != ~0u || i_lo < k0 + 63 || i_hi - k0 > P.l;   // some pair may not be
          uint32_t seen[2] = {there[0], there[1]};      // this row's keys
          if (some_not) {
            if (MODE == DENSE) {
              // 64 remainders a thread, which is what takes the time: 4 x 512 tokens over 2048 to 8192, 12 heads, 1.1 ms (every position 0.12)
#pragma unroll 1
              for (int e = 0; e < 64; ++e)
                if (!near_sees(P.l, pos, k0 + e)) seen[e >> 5] &= ~(1u << (e & 31));
            } else {
              const int last = pos - k0, first = last < 0 ? 0 : last - P.l;     // keys first .. last of the 64
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                const int hi = last - 32 * g, lo = first - 32 * g;
                seen[g] &= hi < 0 ? 0u : hi >= 31 ? ~0u : (2u << hi) - 1u;
                seen[g] &= lo <= 0 ? ~0u : lo > 31 ? 0u : ~0u << lo;
              }
            }
          }
          auto mask = [&](uint32_t (&x)[8], int g) {
            if (some_not) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (!((seen[g >> 2] >> (8 * (g & 3) + e)) & 1u)) x[e] = 0xFF800000u;   // -inf
            }
          };
          // Weights against the reference as it is.  Their sum tells whether a score lies too far above it, which is seldom, so nobody looks for the
          // maximum first (64 comparisons a thread); a row without a reference does
          float sum;
#pragma unroll 1
          for (int pass = 0;; ++pass) {
            const float against = -mst_paged::reference(m);
            const uint64_t nm = pack2(against, against), scale = pack2(P.scale_log2, P.scale_log2);     // two keys an instruction: 6 % less time
            uint64_t add[2] = {0, 0};
            uint32_t x[2][8];
            tmem_ld8_nowait(t_s, x[0]);
#pragma unroll
            for (int g = 0; g < 8; ++g) {
              tmem_ld8_wait(x[g & 1]);
              if (g < 7) tmem_ld8_nowait(t_s + 8u * (g + 1), x[(g + 1) & 1]);
              mask(x[g & 1], g);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint64_t weights = ex2_2(fma2(pack2(x[g & 1][2 * e], x[g & 1][2 * e + 1]), scale, nm));
                add[e & 1] = add2(add[e & 1], weights);
                w[4 * g + e] = pack_bf16_2(weights);
              }
            }
            sum = halves_sum(add2(add[0], add[1]));
            if (pass == 1 || !__any_sync(0xffffffffu, sum > MOST || (live && m == -INFINITY))) break;
            float top = -INFINITY;
#pragma unroll 1
            for (int g = 0; g < 8; ++g) {
              uint32_t x[8];
              tmem_ld8_nowait(t_s + 8u * g, x);
              tmem_ld8_wait(x);
              mask(x, g);
#pragma unroll
              for (int e = 0; e < 8; ++e) top = fmaxf(top, __uint_as_float(x[e]));
            }
            top *= P.scale_log2;
            const bool up = top > m && (sum > MOST || m == -INFINITY);
            const float f = up ? ex2(m - top) : 1.f;       // 0 where nothing has been summed yet
            const bool summed = up && m != -INFINITY;
            if (up) m = top;
            total_w *= f;
            // the outputs so far are complete: the scores of this tile were issued behind the products of the tile before
            if (__any_sync(0xffffffffu, summed)) {
#pragma unroll 1
              for (int g = 0; g < D_; g += 16) {
                uint32_t v[16];
                tmem_ld16_nowait(t_out + (uint32_t)g, v);
                tmem_ld16_wait(v);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                tmem_st16(t_out + (uint32_t)g, v);
              }
            }
          }
          total_w += sum;
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e] = 0u;
        }
        tmem_st32(t_s, w);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * half);
      }
      // the two softmaxes of a row meet: weights 2^(m_k - m), over the sum where the row is complete
      stat[half * 2 * ROWS + r] = m;
      stat[half * 2 * ROWS + ROWS + r] = total_w;
      softmax_warps_meet();
      const float ma = stat[r], mb = stat[2 * ROWS + r];
      const float mm = fmaxf(ma, mb);
      float a0 = ex2(ma - mst_paged::reference(mm)), a1 = ex2(mb - mst_paged::reference(mm));
      const float total = fmaf(a0, stat[ROWS + r], a1 * stat[3 * ROWS + r]);
      if (active == 1) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        a0 *= inv;
        a1 *= inv;
      }
      wait_on(acc_full, lap & 1u, abort_flag);
      const bool ok = __all_sync(0xffffffffu, *abort_flag == 0);
      tc_fence_after();
      const int t = live ? (T.row0 + r) / P.group : 0, h = kvh * P.group + (live ? (T.row0 + r) % P.group : 0);
      const int64_t token = T.first + t, at = ((int64_t)split * P.B.tokens + token) * P.heads + h;
      bool bad = !(total * 0.f == 0.f) || (MODE == NEAR && m1 > m0);     // (a length beyond what the table has room for: see launch)
#pragma unroll
      for (int pc = 0; pc < HALF / 16; ++pc) {
        const int c = half * HALF + pc * 16;
        uint32_t u[16], v[16];
        tmem_ld16_nowait(t_row + OUT0 + (uint32_t)c, u);
        tmem_ld16_nowait(t_row + OUT0 + D_ + (uint32_t)c, v);
        tmem_ld16_wait(u);
        tmem_ld16_wait(v);
        float check = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float o = fmaf(a0, __uint_as_float(u[e]), a1 * __uint_as_float(v[e]));
          check = fmaf(o, 0.f, check);
          u[e] = __float_as_uint(o);
        }
        bad = bad || !(check == 0.f);
        if (active == 1) {
          stage_row(own + (uint32_t)(c / 64) * 2 * TILE_BYTES, r, c % 64, u, 1.f);
        } else if (live && ok) {
#pragma unroll
          for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(P.part_o + at * D_ + c + e) = make_uint4(u[e], u[e + 1], u[e + 2], u[e + 3]);
        }
      }
      tc_fence_before();
      if (live && ok && half == 0) {
        if (active == 1) {
          if (P.lse) P.lse[(int64_t)h * P.B.tokens + token] = (mm + log2f(total)) * LN2;
        } else {
          P.part_m[at * 2] = mm;
          P.part_m[at * 2 + 1] = total;
        }
      }
      const uint32_t redo = __ballot_sync(0xffffffffu, bad && live && ok);
      if (lane == 0 && redo) atomicOr(&again[quarter], redo);
      softmax_warps_meet();
      if (active == 1 && ok) {
#pragma unroll
        for (int it = 0; it < 16; it += 4) {
          const int rr = rs + it + (lane >> 3);
          if (rr < T.rows) {
            __nv_bfloat16* out = P.Out + (int64_t)(T.first + (T.row0 + rr) / P.group) * P.ldo + (int64_t)(kvh * P.group + (T.row0 + rr) % P.group) * D_ + (lane & 7) * 8;
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<uint4*>(out + 64 * q) = lds128(piece_addr(own + q * 2 * TILE_BYTES, rr, lane & 7));
          }
        }
      }
      const bool any = (again[0] | again[1] | again[2] | again[3]) != 0u;
      if (any) {       // seldom: rows that something masked and not finite reached
        softmax_warps_meet();
        for (int rr = warp; rr < T.rows; rr += CW) {
          if (!((again[rr >> 5] >> (rr & 31)) & 1u)) continue;
          float o[D_ / 32], gm, gs;
          const int64_t to_key = (int64_t)key0 + (int64_t)near * KEYS;
          const int64_t tk = T.first + (T.row0 + rr) / P.group;
          const int hh = kvh * P.group + (T.row0 + rr) % P.group;
          row_again<D_>(P, b, (int)tk, hh, T.p_lo + (T.row0 + rr) / P.group - T.t_lo, key0, have < to_key ? have : (int)to_key, P.l, MODE == DENSE, m0, m1, o,
                        gm, gs);
          if (active == 1) {
            finish<D_ / 32>(P, tk, hh, lane, o, gm, gs);
          } else {
            const int64_t to = ((int64_t)split * P.B.tokens + tk) * P.heads + hh;
#pragma unroll
            for (int e = 0; e < D_ / 32; ++e) P.part_o[to * D_ + lane * (D_ / 32) + e] = o[e];
            if (lane == 0) {
              P.part_m[to * 2] = gm;
              P.part_m[to * 2 + 1] = gs;
            }
          }
        }
        softmax_warps_meet();
        if (warp == 0 && lane < ROWS / 32) again[lane] = 0u;
      }
      fence_async_smem();           // the own rows' place is written by the next tile's copy
    }
    if (__syncthreads_or(*abort_flag != 0)) break;        // everybody is done with this tile of rows
    ++lap;
    if (MODE == FAR && m1 > m0) ++far_lap;
    base_t += (uint32_t)near;
  }
  if (*abort_flag) {
    for (int t = 0; t < 2000; ++t) __nanosleep(1000);   // let copies and products in flight land
  }
  tc_fence_before();
  __syncthreads();
  if (warp == CW + 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM_COLS) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------- maps and launch
bool encode(CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  mst_encode_tiled_fn fn = mst_encode_tiled();
  if (!fn) return false;
  const cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// rows of a box: the largest power of two up to 64 that divides a page
int box_rows(int page_size) {
  int r = 1;
  while (r < TS && page_size % (2 * r) == 0) r *= 2;
  return r;
}
// The cache as (values, then slots, heads and pages with the closest first); a dimension of one has whatever stride fits
bool cache_maps(const Params& P, TileParams& A, CUtensorMap* tmK, CUtensorMap* tmV, int box) {
  struct Dim { int what; int64_t n, stride; };
  Dim d[3] = {{0, P.C.page_size, P.C.token_stride}, {1, P.C.kv_heads, P.C.head_stride}, {2, P.C.num_pages, P.C.page_stride}};
  int64_t widest = P.C.D;
  for (const Dim& x : d)
    if (x.n > 1 && x.stride > widest) widest = x.stride;
  for (Dim& x : d)
    if (x.n <= 1) { x.n = 1; x.stride = widest; }
  for (int i = 0; i < 2; ++i)
    for (int k = 0; k < 2; ++k)
      if (d[k + 1].stride < d[k].stride) { const Dim t = d[k]; d[k] = d[k + 1]; d[k + 1] = t; }
  cuuint64_t dims[4] = {(cuuint64_t)P.C.D, 1, 1, 1}, strides[3];
  cuuint32_t boxes[4] = {64u, 1u, 1u, 1u};
  for (int i = 0; i < 3; ++i) {
    dims[i + 1] = (cuuint64_t)d[i].n;
    strides[i] = (cuuint64_t)d[i].stride * 2;
    if (strides[i] >= (1ULL << 40)) return false;
    if (d[i].what == 0) { A.at_slot = i + 1; boxes[i + 1] = (cuuint32_t)box; }
    if (d[i].what == 1) A.at_head = i + 1;
    if (d[i].what == 2) A.at_page = i + 1;
  }
  return encode(tmK, P.C.K, 4, dims, strides, boxes) && encode(tmV, P.C.V, 4, dims, strides, boxes);
}

template <int D_, Mode MODE>
mst_status_t launch(const TileParams& A, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s) {
  MST_SMEM_LIMIT((paged_tiles_kernel<D_, MODE>), Shape<D_>::SMEM);
  const dim3 grid((unsigned)(A.P.C.kv_heads * A.P.splits), (unsigned)A.P.B.batch, (unsigned)A.count);
  MST_CUDA_TRY(mst_launch_overlapped(paged_tiles_kernel<D_, MODE>, grid, dim3(THREADS), Shape<D_>::SMEM, s, tmQ, tmK, tmV, A));
  return MST_OK;
}
template <int D_>
mst_status_t launch(const TileParams& A, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, cudaStream_t s) {
  const int64_t reach = (int64_t)A.P.B.table_stride * A.P.C.page_size;
  if (A.P.l < DENSE_BELOW) return launch<D_, DENSE>(A, tmQ, tmK, tmV, s);
  // lengths beyond the table's room may still have rows two strides in, which are formed again key by key
  return reach / 2 < A.P.l ? launch<D_, NEAR>(A, tmQ, tmK, tmV, s) : launch<D_, FAR>(A, tmQ, tmK, tmV, s);
}

}  // namespace

namespace mst_paged {
mst_status_t launch_tiles(const Params& P, const Plan& plan, cudaStream_t s) {
  TileParams A = {};
  A.P = P;
  A.rows = plan.rows;
  A.by_tokens = Divider::of((uint32_t)(plan.rows / P.group));
  A.per_token = (float)P.group / (float)plan.rows;
  A.count = plan.count;
  CUtensorMap tmQ, tmK = {}, tmV = {};
  const cuuint64_t dims[3] = {(cuuint64_t)P.C.D, (cuuint64_t)P.heads, (cuuint64_t)P.B.tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)P.C.D * 2, (cuuint64_t)P.ldq * 2};
  const cuuint32_t boxes[3] = {64u, (cuuint32_t)P.group, (cuuint32_t)(plan.rows / P.group)};
  if (strides[1] >= (1ULL << 40) || !encode(&tmQ, P.Q, 3, dims, strides, boxes)) return MST_ERR_SHAPE;
  const int box = box_rows(P.C.page_size);
  A.box = box >= 8 && P.C.num_pages > 0 && cache_maps(P, A, &tmK, &tmV, box) ? box : 0;
  if (A.box == 0) tmK = tmV = tmQ;       // not read, but fetched ahead
  return P.C.D == 64 ? launch<64>(A, tmQ, tmK, tmV, s) : launch<128>(A, tmQ, tmK, tmV, s);
}
}  // namespace mst_paged

mst_status_t mst_paged_tiles_error_flags(int32_t* flags) {
  int32_t bad = 0, rows = 0;
  int v = 0;
  MST_TRY(mst_paged::take_flag((const void*)&mst_paged::g_bad_page, &bad));
  MST_TRY(mst_paged::take_flag((const void*)&mst_paged::g_bad_rows, &rows));
  MST_CUDA_TRY(cudaMemcpyFromSymbol(&v, g_wait_error, sizeof(int)));
  *flags = bad | (v << 1) | (rows << 2);
  return MST_OK;
}
