// Norm and rotation of one head's row by a group of lanes: shared by the training calls and the append to a paged cache.
//
// A row of D = 8 .. 256 values lies in the registers of G neighbouring lanes, four pairs (u, v) a lane: two runs of four values, `near` and
// `far` elements into the row.  Where pairs are halves apart the runs are rot / 2 apart, so both values of a pair are in one lane and nothing
// is exchanged but the sum of squares (log2 G shuffles); neighbouring pairs lie within a run.  Values that do not turn fill further lanes
// with runs of their own.  Two values that go through the same step share an instruction (f32x2).  With c, s the cosine and sine of the
// pair's angle and r = 1 / sqrt(mean(x^2) + eps)
//   u' = r (u gamma_u c - v gamma_v s),   v' = r (u gamma_u s + v gamma_v c)
// where the products of weights and angles change with the token and the side (queries, keys) only, not from head to head.
#pragma once
#include <cuda_bf16.h>

#include "mst_internal.cuh"
#include "mst_tc_gemm.cuh"
#include "mst_tc_ptx.cuh"

namespace mst_rot {
using namespace mst_ptx;

constexpr int WARPS = 8;                    // of a block, each on its own
constexpr int MAX_HALF = 128;               // rot_dim / 2

struct Rotation {
  int D, rot, inter;
  float eps;
  const float *inv_freq, *gamma_q, *gamma_k;
};

inline mst_status_t check(const mst_rotation_t* r, Rotation* out) {
  if (!r) return MST_ERR_INVALID_ARG;
  if (r->head_dim < 8 || r->head_dim > 256 || r->head_dim % 8 != 0) return MST_ERR_SHAPE;
  if (r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 16 != 0) return MST_ERR_SHAPE;
  if (r->rot_dim > 0 && !r->inv_freq) return MST_ERR_INVALID_ARG;
  if (!(r->eps >= 0.f)) return MST_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(r->inv_freq) & 3u) != 0) return MST_ERR_SHAPE;
  if (((reinterpret_cast<uintptr_t>(r->gamma_q) | reinterpret_cast<uintptr_t>(r->gamma_k)) & 15u) != 0) return MST_ERR_SHAPE;
  *out = Rotation{r->head_dim, r->rot_dim, r->interleaved != 0, r->eps, r->inv_freq, r->gamma_q, r->gamma_k};
  return MST_OK;
}
// lanes of a row: D / 8 of them have values; rows of up to 32 values share a kernel
inline int lanes_of(int D) { return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32; }

// ---------------------------------------------------------------------------------------------- a lane's part of a row
struct Lane {
  int near, far;    // first elements of its two runs
  bool in, turns;
  __device__ __forceinline__ Lane(const Rotation& R, int li, bool inter) {
    in = 8 * li < R.D;
    turns = 8 * li < R.rot;
    if (inter) {
      near = 8 * li;
      far = near + 4;
    } else if (turns) {
      near = 4 * li;
      far = near + R.rot / 2;
    } else {
      near = R.rot + 4 * (li - R.rot / 8);
      far = near + (R.D - R.rot) / 2;
    }
    if (!in) near = far = 0;
  }
};
template <typename T>
struct Raw {
  uint32_t w[sizeof(T) * 2];
};
__device__ __forceinline__ void load_row(Raw<__nv_bfloat16>& r, const __nv_bfloat16* p, const Lane& L) {
  const uint2 a = *reinterpret_cast<const uint2*>(p + L.near), b = *reinterpret_cast<const uint2*>(p + L.far);
  r.w[0] = a.x; r.w[1] = a.y; r.w[2] = b.x; r.w[3] = b.y;
}
__device__ __forceinline__ void load_row(Raw<float>& r, const float* p, const Lane& L) {
  const uint4 a = *reinterpret_cast<const uint4*>(p + L.near), b = *reinterpret_cast<const uint4*>(p + L.far);
  r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
  r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
}
__device__ __forceinline__ void store_row(const Raw<__nv_bfloat16>& r, __nv_bfloat16* p, const Lane& L) {
  *reinterpret_cast<uint2*>(p + L.near) = make_uint2(r.w[0], r.w[1]);
  *reinterpret_cast<uint2*>(p + L.far) = make_uint2(r.w[2], r.w[3]);
}
__device__ __forceinline__ void store_row(const Raw<float>& r, float* p, const Lane& L) {
  *reinterpret_cast<uint4*>(p + L.near) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
  *reinterpret_cast<uint4*>(p + L.far) = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
}
template <typename T>
__device__ __forceinline__ void no_row(Raw<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) * 2; ++i) r.w[i] = 0u;
}

// Four pairs, two to a register pair: u and v hold values 0, 1 and 2, 3
struct Pairs {
  uint64_t u[2], v[2];
};
// eight values in the order of memory (two runs of four) <-> pairs
template <bool INTER>
__device__ __forceinline__ Pairs pairs_of(const float (&x)[8]) {
  Pairs p;
  if (INTER) {
    p.u[0] = pack2(x[0], x[2]); p.v[0] = pack2(x[1], x[3]);
    p.u[1] = pack2(x[4], x[6]); p.v[1] = pack2(x[5], x[7]);
  } else {
    p.u[0] = pack2(x[0], x[1]); p.u[1] = pack2(x[2], x[3]);
    p.v[0] = pack2(x[4], x[5]); p.v[1] = pack2(x[6], x[7]);
  }
  return p;
}
template <bool INTER>
__device__ __forceinline__ void values_of(const Pairs& p, float (&x)[8]) {
  if (INTER) {
    unpack2(p.u[0], x[0], x[2]); unpack2(p.v[0], x[1], x[3]);
    unpack2(p.u[1], x[4], x[6]); unpack2(p.v[1], x[5], x[7]);
  } else {
    unpack2(p.u[0], x[0], x[1]); unpack2(p.u[1], x[2], x[3]);
    unpack2(p.v[0], x[4], x[5]); unpack2(p.v[1], x[6], x[7]);
  }
}
template <bool INTER>
__device__ __forceinline__ Pairs widen(const Raw<__nv_bfloat16>& r) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.w[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
  }
  return pairs_of<INTER>(x);
}
template <bool INTER>
__device__ __forceinline__ Pairs widen(const Raw<float>& r) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.w[i]);
  return pairs_of<INTER>(x);
}
template <bool INTER>
__device__ __forceinline__ void narrow(const Pairs& p, Raw<__nv_bfloat16>& r) {
  float x[8];
  values_of<INTER>(p, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
}
template <bool INTER>
__device__ __forceinline__ void narrow(const Pairs& p, Raw<float>& r) {
  float x[8];
  values_of<INTER>(p, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(x[i]);
}
// a lane's norm weights (ones where there is no norm or no value)
template <bool INTER>
__device__ __forceinline__ Pairs weights(const float* gamma, const Lane& L) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = 1.f;
  if (gamma && L.in) {
    const float4 a = *reinterpret_cast<const float4*>(gamma + L.near), b = *reinterpret_cast<const float4*>(gamma + L.far);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  return pairs_of<INTER>(x);
}
__device__ __forceinline__ float halves_sum(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
__device__ __forceinline__ float dot(const Pairs& a, const Pairs& b) {
  return halves_sum(add2(fma2(a.u[0], b.u[0], mul2(a.v[0], b.v[0])), fma2(a.u[1], b.u[1], mul2(a.v[1], b.v[1]))));
}
template <int G>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = 1; o < G; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---------------------------------------------------------------------------------------------- the turn
// Cosines and sines of a position into a warp's own table, and out of it those of the lane's pairs.  The angle in turns, position * inv_freq /
// 2 pi, is formed in fp64 and loses its whole part there: 53 bits hold 2^31 turns to 2^-22, and what is left goes to sincospi in fp32.
struct Turn {
  uint64_t c[2], s[2];
};
template <bool INTER>
__device__ __forceinline__ Turn turn_of(float2* table, const Rotation& R, const Lane& L, int pos, int lane) {
  __syncwarp();
  for (int i = lane; i < R.rot / 2; i += 32) {
    const double turns = (double)pos * ((double)R.inv_freq[i] * 0.15915494309189533577);
    float2 v;
    sincospif((float)(2.0 * (turns - rint(turns))), &v.y, &v.x);
    table[i] = v;
  }
  __syncwarp();
  Turn t;
  t.c[0] = t.c[1] = pack2(1.f, 1.f);
  t.s[0] = t.s[1] = 0ULL;
  if (L.turns) {
    const float4* at = reinterpret_cast<const float4*>(table + (INTER ? L.near / 2 : L.near));
    const float4 a = at[0], b = at[1];
    t.c[0] = pack2(a.x, a.z); t.s[0] = pack2(a.y, a.w);
    t.c[1] = pack2(b.x, b.z); t.s[1] = pack2(b.y, b.w);
  }
  return t;
}
__device__ __forceinline__ uint64_t negated(uint64_t v) { return v ^ 0x8000000080000000ULL; }

// A warp's steps through a token: 32 / G rows each, first the queries', then the keys', then the values' (which are only carried along).
struct Steps {
  int q, k, v;
  __host__ __device__ Steps(int rows, int hq, int hk, int hv) : q((hq + rows - 1) / rows), k((hk + rows - 1) / rows), v((hv + rows - 1) / rows) {}
  __host__ __device__ int all() const { return q + k + v; }
};
// Tokens alone fill the GPU from some thousands on; below that a token's steps are shared out, so that a few tokens are not a few warps' long
// chains of loads.  Returns the warps of a token and sets their steps.
inline int share_token(int64_t tokens, int steps, int* per_warp) {
  const int64_t want = (int64_t)mst_sm_count() * 24 / (tokens > 0 ? tokens : 1);
  const int warps = want <= 1 ? 1 : want >= steps ? steps : (int)want;
  *per_warp = (steps + warps - 1) / warps;
  return (steps + *per_warp - 1) / *per_warp;
}

}  // namespace mst_rot
