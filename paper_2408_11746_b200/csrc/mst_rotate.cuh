// Norm and rotation of one head's row by a group of lanes: shared by the training calls and the append to a paged cache.
//
// A row of D = 8 .. 256 values lies in the registers of G neighbouring lanes, 2 N pairs (u, v) a lane (N = 4 forward, 2 in the gradients, which hold
// twice as much): two runs of 2 N values, `near` and `far` elements into the row.  Where pairs are halves apart the runs are rot / 2 apart, so both values of a pair are in one lane and nothing
// is exchanged but the sum of squares (log2 G shuffles); neighbouring pairs lie within a run.  Values that do not turn fill further lanes
// with runs of their own.  Two values that go through the same step share an instruction (f32x2).  With c, s the cosine and sine of the
// pair's angle and r = 1 / sqrt(mean(x^2) + eps)
//   u' = r (u gamma_u c - v gamma_v s),   v' = r (u gamma_u s + v gamma_v c)
// A group of lanes keeps to one side, queries or keys, so the products of weights and angles are formed once a token.  (With eight values a lane
// and groups that changed sides, a token of 24 rows took 1156 instructions, which was what 16384 of them waited for: 29 us.)
#pragma once
#include <cuda_bf16.h>

#include "mst_angle.h"
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
// lanes of a row: D / (4 N) of them have values; rows of up to 32 values share a kernel
inline int lanes_of(int D, int N) { return (D <= 32 ? 8 : D <= 64 ? 16 : D <= 128 ? 32 : 64) / N; }

// ---------------------------------------------------------------------------------------------- a lane's part of a row
struct Lane {
  int near, far;    // first elements of its two runs of `run`
  bool in, in_far, turns;
  __device__ __forceinline__ Lane(const Rotation& R, int li, bool inter, int run) {
    in = 2 * run * li < R.D;
    turns = 2 * run * li < R.rot;
    if (!inter && turns) {
      near = run * li;
      far = near + R.rot / 2;
    } else {
      near = 2 * run * li;
      far = near + run;
    }
    if (!in) near = far = 0;
    in_far = in && far < R.D;
    if (!in_far) far = near;
  }
};
template <typename T, int N>
struct Raw {
  uint32_t w[sizeof(T) * N];
};
// a run of 2 N values: 8 bytes or 16 at a time
template <int WORDS>
__device__ __forceinline__ void load_run(uint32_t* w, const void* p) {
  if (WORDS == 2) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x; w[1] = a.y;
  } else {
#pragma unroll
    for (int i = 0; i + 4 <= WORDS; i += 4) {
      const uint4 a = reinterpret_cast<const uint4*>(p)[i / 4];
      w[i] = a.x; w[i + 1] = a.y; w[i + 2] = a.z; w[i + 3] = a.w;
    }
  }
}
template <int WORDS>
__device__ __forceinline__ void store_run(const uint32_t* w, void* p) {
  if (WORDS == 2) {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i + 4 <= WORDS; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  }
}
template <typename T, int N>
__device__ __forceinline__ void load_row(Raw<T, N>& r, const T* p, const Lane& L) {
  constexpr int W = sizeof(T) * N / 2;
  load_run<W>(r.w, p + L.near);
  if (L.in_far) load_run<W>(r.w + W, p + L.far);
}
template <typename T, int N>
__device__ __forceinline__ void store_row(const Raw<T, N>& r, T* p, const Lane& L) {
  constexpr int W = sizeof(T) * N / 2;
  store_run<W>(r.w, p + L.near);
  if (L.in_far) store_run<W>(r.w + W, p + L.far);
}
template <typename T, int N>
__device__ __forceinline__ void no_row(Raw<T, N>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) * N; ++i) r.w[i] = 0u;
}

// 2 N pairs, two to a register pair
template <int N>
struct Pairs {
  uint64_t u[N], v[N];
};
// 4 N values in the order of memory (two runs) <-> pairs
template <bool INTER, int N>
__device__ __forceinline__ Pairs<N> pairs_of(const float (&x)[4 * N]) {
  Pairs<N> p;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (INTER) {
      p.u[k] = pack2(x[4 * k], x[4 * k + 2]);
      p.v[k] = pack2(x[4 * k + 1], x[4 * k + 3]);
    } else {
      p.u[k] = pack2(x[2 * k], x[2 * k + 1]);
      p.v[k] = pack2(x[2 * N + 2 * k], x[2 * N + 2 * k + 1]);
    }
  }
  return p;
}
template <bool INTER, int N>
__device__ __forceinline__ void values_of(const Pairs<N>& p, float (&x)[4 * N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (INTER) {
      unpack2(p.u[k], x[4 * k], x[4 * k + 2]);
      unpack2(p.v[k], x[4 * k + 1], x[4 * k + 3]);
    } else {
      unpack2(p.u[k], x[2 * k], x[2 * k + 1]);
      unpack2(p.v[k], x[2 * N + 2 * k], x[2 * N + 2 * k + 1]);
    }
  }
}
template <bool INTER, int N>
__device__ __forceinline__ Pairs<N> widen(const Raw<__nv_bfloat16, N>& r) {
  float x[4 * N];
#pragma unroll
  for (int i = 0; i < 2 * N; ++i) {
    x[2 * i] = __uint_as_float(r.w[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
  }
  return pairs_of<INTER, N>(x);
}
template <bool INTER, int N>
__device__ __forceinline__ Pairs<N> widen(const Raw<float, N>& r) {
  float x[4 * N];
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) x[i] = __uint_as_float(r.w[i]);
  return pairs_of<INTER, N>(x);
}
template <bool INTER, int N>
__device__ __forceinline__ void narrow(const Pairs<N>& p, Raw<__nv_bfloat16, N>& r) {
  float x[4 * N];
  values_of<INTER, N>(p, x);
#pragma unroll
  for (int i = 0; i < 2 * N; ++i) r.w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
}
template <bool INTER, int N>
__device__ __forceinline__ void narrow(const Pairs<N>& p, Raw<float, N>& r) {
  float x[4 * N];
  values_of<INTER, N>(p, x);
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) r.w[i] = __float_as_uint(x[i]);
}
// a lane's norm weights (ones where there is no norm or no value)
template <bool INTER, int N>
__device__ __forceinline__ Pairs<N> weights(const float* gamma, const Lane& L) {
  float x[4 * N];
#pragma unroll
  for (int e = 0; e < 4 * N; ++e) x[e] = 1.f;
  if (gamma && L.in) {
#pragma unroll
    for (int i = 0; i < 2 * N; i += 4) {
      const float4 a = *reinterpret_cast<const float4*>(gamma + L.near + i), b = *reinterpret_cast<const float4*>(gamma + L.far + i);
      x[i] = a.x; x[i + 1] = a.y; x[i + 2] = a.z; x[i + 3] = a.w;
      x[2 * N + i] = b.x; x[2 * N + i + 1] = b.y; x[2 * N + i + 2] = b.z; x[2 * N + i + 3] = b.w;
    }
  }
  return pairs_of<INTER, N>(x);
}
__device__ __forceinline__ float halves_sum(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
template <int N>
__device__ __forceinline__ float dot(const Pairs<N>& a, const Pairs<N>& b) {
  uint64_t s = mul2(a.u[0], b.u[0]), t = mul2(a.v[0], b.v[0]);
#pragma unroll
  for (int k = 1; k < N; ++k) {
    s = fma2(a.u[k], b.u[k], s);
    t = fma2(a.v[k], b.v[k], t);
  }
  return halves_sum(add2(s, t));
}
template <int G>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = 1; o < G; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---------------------------------------------------------------------------------------------- the turn
// Cosines and sines of a position into a warp's own table, and out of it those of the lane's pairs.  An angle loses its whole turns before it is
// rounded (mst_angle.h); what is left goes to sincospi in fp32, off by 2^-25 of half a turn at most: 1e-7.
// A lane keeps the frequencies that it sees to: lane, lane + 32, .. of rot / 2; K of them are enough for the longest row of G lanes.
template <int G, int N>
struct Frequencies {
  static constexpr int K = 2 * G * N <= 32 ? 1 : 2 * G * N / 32;
  float f[K];
  __device__ __forceinline__ Frequencies(const Rotation& R, int lane) {
#pragma unroll
    for (int k = 0; k < K; ++k) f[k] = lane + 32 * k < R.rot / 2 ? R.inv_freq[lane + 32 * k] : 0.f;
  }
};
// for all positions: made where nothing else is to be asked of memory any more (ahead of the lookup of rows to append 3 % of their time)
template <int G, int N>
struct Steps {
  uint64_t step[Frequencies<G, N>::K];
  uint32_t none = 0;          // bits: frequencies that are no finite numbers
  __device__ __forceinline__ explicit Steps(const Frequencies<G, N>& F) {
#pragma unroll
    for (int k = 0; k < Frequencies<G, N>::K; ++k) {
      step[k] = step_of(F.f[k]);
      if (!(F.f[k] - F.f[k] == 0.f)) none |= 1u << k;
    }
  }
};
template <int N>
struct Turn {
  uint64_t c[N], s[N];
};
template <bool INTER, int G, int N>
__device__ __forceinline__ Turn<N> turn_of(float2* table, const Rotation& R, const Steps<G, N>& S, const Lane& L, int pos, int lane) {
  __syncwarp();
#pragma unroll
  for (int k = 0; k < Frequencies<G, N>::K; ++k) {
    if (32 * k >= R.rot / 2) break;
    float2 v;
    sincospif((S.none >> k) & 1u ? NAN : half_turns(S.step[k], pos), &v.y, &v.x);
    table[lane + 32 * k] = v;
  }
  __syncwarp();
  Turn<N> t;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    t.c[k] = pack2(1.f, 1.f);
    t.s[k] = 0ULL;
  }
  if (L.turns) {
    const float4* at = reinterpret_cast<const float4*>(table + (INTER ? L.near / 2 : L.near));
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float4 a = at[k];
      t.c[k] = pack2(a.x, a.z);
      t.s[k] = pack2(a.y, a.w);
    }
  }
  return t;
}
__device__ __forceinline__ uint64_t negated(uint64_t v) { return v ^ 0x8000000080000000ULL; }

// A warp's groups of lanes: the first `q` take the queries' rows in turn, the others the keys', as many of each as make the fewest steps.
struct Groups {
  int q, steps;
};
inline Groups groups_of(int lanes, int hq, int hk) {
  const int all = 32 / lanes;
  if (hq == 0 || hk == 0) return Groups{hq == 0 ? 0 : all, (hq + hk + all - 1) / all};
  Groups best = {0, 1 << 30};
  for (int q = 1; q < all; ++q) {
    const int a = (hq + q - 1) / q, b = (hk + all - q - 1) / (all - q), steps = a > b ? a : b;
    if (steps < best.steps) best = Groups{q, steps};
  }
  return best;
}
// Tokens alone fill the GPU from some thousands on; below that a token's steps are shared out, so that a few tokens are not a few warps' long
// chains of loads.  Returns the warps of a token and sets their steps.
inline int share_token(int64_t tokens, int steps, int* per_warp) {
  const int64_t want = (int64_t)mst_sm_count() * 24 / (tokens > 0 ? tokens : 1);
  const int warps = want <= 1 ? 1 : want >= steps ? steps : (int)want;
  *per_warp = (steps + warps - 1) / warps;
  return (steps + *per_warp - 1) / *per_warp;
}

}  // namespace mst_rot
