// Norm and rotation of one head's row by a group of lanes: shared by the training calls and the append to a paged cache.
//
// A row of D = 8 .. 256 values lies in the registers of D / 8 neighbouring lanes, eight values a lane: one 16-byte load (bf16) or two
// (fp32), and the sum of squares is log2(lanes) shuffles.  With c, s the cosine and sine of a value's angle, and a partner value p,
//   y = r (x A + p B),   A = gamma c,  B = -/+ gamma_partner s,   r = 1 / sqrt(mean(x^2) + eps)
// so a row costs two multiply-adds a value once A and B are in registers; they change with the token and the side only (queries, keys),
// not from head to head.  The partner is in the lane itself (neighbouring pairs) or, raw, one shuffle a word away (halves).
#pragma once
#include <cuda_bf16.h>

#include "mst_internal.cuh"
#include "mst_tc_gemm.cuh"

namespace mst_rot {

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
// lanes of a row: the power of two that holds D / 8
inline int lanes_of(int D) {
  int g = 1;
  while (g * 8 < D) g *= 2;
  return g;
}

// ---------------------------------------------------------------------------------------------- eight values of a row
template <typename T>
struct Raw {
  static constexpr int W = sizeof(T) * 2;   // words
  uint32_t w[W];
};
template <typename T>
__device__ __forceinline__ Raw<T> load8(const T* p) {
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < Raw<T>::W; i += 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
    r.w[i] = v.x; r.w[i + 1] = v.y; r.w[i + 2] = v.z; r.w[i + 3] = v.w;
  }
  return r;
}
template <typename T>
__device__ __forceinline__ Raw<T> zero8() {
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < Raw<T>::W; ++i) r.w[i] = 0u;
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Raw<T>& r) {
#pragma unroll
  for (int i = 0; i < Raw<T>::W; i += 4)
    *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(p) + i) = make_uint4(r.w[i], r.w[i + 1], r.w[i + 2], r.w[i + 3]);
}
__device__ __forceinline__ void widen(const Raw<__nv_bfloat16>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.w[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void widen(const Raw<float>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.w[i]);
}
__device__ __forceinline__ void narrow(const float (&x)[8], Raw<__nv_bfloat16>& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    r.w[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
}
__device__ __forceinline__ void narrow(const float (&x)[8], Raw<float>& r) {
#pragma unroll
  for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(x[i]);
}
template <int G>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = 1; o < G; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---------------------------------------------------------------------------------------------- the turn
// Cosines and sines of a position into a warp's own table.  The angle in turns, position * inv_freq / 2 pi, is formed in fp64 and loses its whole
// part there: 53 bits hold 2^31 turns to 2^-22, and what is left goes to sincospi in fp32.
__device__ __forceinline__ void angles(float2* table, const Rotation& R, int pos, int lane) {
  __syncwarp();
  for (int i = lane; i < R.rot / 2; i += 32) {
    const double turns = (double)pos * ((double)R.inv_freq[i] * 0.15915494309189533577);
    float2 v;
    sincospif((float)(2.0 * (turns - rint(turns))), &v.y, &v.x);
    table[i] = v;
  }
  __syncwarp();
}
// What a lane's eight values are turned by: y = c x + s p with p the partner's value
struct Turn {
  float c[8], s[8];
};
// the place of a lane in its row
struct Lane {
  int e0;        // first value
  int from;      // the lane that holds the partners (halves)
  bool turns;    // e0 < rot
  bool first;    // halves: the a of the pairs
  __device__ __forceinline__ Lane(const Rotation& R, int li, int lane) : e0(8 * li), from(lane), turns(8 * li < R.rot), first(8 * li < R.rot / 2) {
    if (!R.inter && turns) from = first ? lane + R.rot / 16 : lane - R.rot / 16;
  }
};
__device__ __forceinline__ Turn turn_of(const Rotation& R, const Lane& L, const float2* table, bool back) {
  Turn t;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t.c[e] = 1.f;
    t.s[e] = 0.f;
  }
  if (L.turns) {
    const float flip = back ? -1.f : 1.f;
    if (R.inter) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 v = table[L.e0 / 2 + e / 2];
        t.c[e] = v.x;
        t.s[e] = (e & 1) ? flip * v.y : -flip * v.y;
      }
    } else {
      const int i0 = L.first ? L.e0 : L.e0 - R.rot / 2;
      const float sign = L.first ? -flip : flip;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 v = table[i0 + e];
        t.c[e] = v.x;
        t.s[e] = sign * v.y;
      }
    }
  }
  return t;
}
// the partners' values
template <typename T>
__device__ __forceinline__ void partners(const Rotation& R, const Lane& L, const Raw<T>& raw, const float (&x)[8], float (&p)[8]) {
  if (R.inter) {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = x[e ^ 1];
  } else {
    Raw<T> o;
#pragma unroll
    for (int i = 0; i < Raw<T>::W; ++i) o.w[i] = __shfl_sync(0xffffffffu, raw.w[i], L.from);
    widen(o, p);
  }
}
// A and B of a side: the turn with the weights in it (weights of values beyond D and of no norm: 1)
__device__ __forceinline__ void weights(const Rotation& R, const Lane& L, const float* gamma, float (&own)[8], float (&partner)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) own[e] = partner[e] = 1.f;
  if (gamma && L.e0 < R.D) {
#pragma unroll
    for (int e = 0; e < 8; ++e) own[e] = gamma[L.e0 + e];
    if (L.turns) {
      const int at = R.inter ? L.e0 : L.first ? L.e0 + R.rot / 2 : L.e0 - R.rot / 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) partner[e] = gamma[R.inter ? at + (e ^ 1) : at + e];
    }
  }
}

// A warp's steps through a token: 32 / G rows each, first the queries', then the keys', then the values' (which are only carried along).
struct Steps {
  int q, k, v;
  __host__ __device__ Steps(int rows, int hq, int hk, int hv) : q((hq + rows - 1) / rows), k((hk + rows - 1) / rows), v((hv + rows - 1) / rows) {}
  __host__ __device__ int all() const { return q + k + v; }
};
// Tokens alone fill the GPU from some thousands on; below that a token's steps are shared out, so that a few tokens are not a few warps' long
// chains of loads.
inline int warps_of_token(int64_t tokens, int steps) {
  const int64_t want = (int64_t)mst_sm_count() * 32 / (tokens > 0 ? tokens : 1);
  return want <= 1 ? 1 : want >= steps ? (steps > 0 ? steps : 1) : (int)want;
}

}  // namespace mst_rot
