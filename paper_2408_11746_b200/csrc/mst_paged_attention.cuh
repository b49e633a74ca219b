// Shared by the two forms of the attention over a paged cache: parameters, results of a row, a row formed again.
#pragma once
#include <cuda_bf16.h>

#include "mst_attention_tile.cuh"
#include "mst_internal.cuh"
#include "mst_paged.cuh"

namespace mst_paged {
using namespace mst_ptx;
using mst_att::ex2;

static __device__ int g_bad_page = 0, g_bad_rows = 0;     // each file's own

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
  Divider by_group, by_l, by_least;
  float scale_log2;
  int splits, least;      // most ranges of a list, and the least units of one (plan)
  float* part_o;          // [splits][tokens * heads][D]: sums against part_m, [splits][tokens * heads][2]: reference and sum of weights
  float* part_m;
};

constexpr int UNIT = 64;  // keys of a list that stay together

// A tile of sequence b (mst_paged_list.h)
__device__ __forceinline__ bool locate(List& T, const Params& P, int b, int tile, int R) {
  const RowsOf rows(P.B.first[b], P.B.first[b + 1], P.B.len[b], P.B.tokens);
  const int64_t reach = (int64_t)P.B.table_stride * P.C.page_size;
  if (rows.outside) g_bad_rows = 1;
  if (!T.locate(rows.first, rows.end, rows.len, P.B.tokens, P.by_group, P.by_l, reach, tile, R)) return false;
  if (rows.len > reach) g_bad_page = 1;
  return true;
}

// 16 bytes, of which `size` (16 or none) come from src, which lies in the cache either way, and the others are zero
__device__ __forceinline__ void cp16_of(uint32_t dst, const void* src, uint32_t size) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) { cp16_of(dst, src, there ? 16u : 0u); }
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

// A row whose sums are not finite, formed again by one warp over the keys it looks at alone: what the matrix products multiplied by a weight
// of zero may have been infinite or NaN.  The row of token row `row`, head h, position pos; keys: positions from .. to - 1 at distances up to
// `window` (every: and at multiples of the stride), and the strided ones m_from .. m_to - 1 steps back.  Lane: D / 32 neighbouring columns.
template <int D>
static __device__ __noinline__ void row_again(const Params& P, int b, int row, int h, int pos, int from, int to, int window, bool every, int m_from,
                                              int m_to, float (&o)[D / 32], float& m, float& sum) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const __nv_bfloat16* q = P.Q + (int64_t)row * P.ldq + (int64_t)h * D + lane * E;
  m = -INFINITY;
  sum = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  auto add = [&](int j) {
    const Slot s = slot_of(P.C, P.B, b, j, &g_bad_page);
    if (!s.exists) return;
    const int64_t at = s.at + (int64_t)(h / P.group) * P.C.head_stride + lane * E;
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
  };
  for (int j = from; j < to && j <= pos; ++j)
    if (pos - j <= window || (every && (pos - j) % P.l == 0)) add(j);
  for (int k = m_from; k < m_to; ++k) {
    const int64_t j = (int64_t)pos - (int64_t)k * P.l;
    if (j < 0) break;
    add((int)j);
  }
}

struct Plan {
  bool tiles;             // 128-row tiles on the tensor cores, otherwise few rows
  int rows;               // of a tile
  int count;              // tiles of a sequence in the grid
  int splits, least;
};
// the form for many rows (mst_paged_tiles.cu); MST_ERR_SHAPE where the queries cannot be described to the TMA unit
mst_status_t launch_tiles(const Params& P, const Plan& plan, cudaStream_t s);

}  // namespace mst_paged
