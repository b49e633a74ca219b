// Norm of queries and keys for each head with the position rotation in the same pass: forward, gradients, and the form that
// appends to a paged cache.  The arithmetic of a row is in mst_rotate.cuh; the kernels differ in where rows come from and go to.
//
// Bound: HBM (each row is read once and written once), or a launch and a trip to memory where there are few tokens.  A warp takes a token (or
// a share of its heads) and has the loads of four steps in flight before it works out the angles; no block-wide step anywhere.
#include "mst_paged.cuh"
#include "mst_rotate.cuh"

namespace {
using namespace mst_rot;

__device__ int g_bad_page = 0;

struct RowsParams {
  Rotation R;
  const void *Q, *K, *V;
  void *Qo, *Ko;
  int64_t ld, ldq;
  int hq, hk;
  const int32_t* positions;
  int seq_len;
  int64_t tokens;
  int share, per_warp;         // warps of a token, steps of a warp
  mst_paged::Cache cache;
  mst_paged::Batch batch;
};

constexpr int AHEAD = 4;       // steps whose loads are in flight together

template <typename T, int G, bool APPEND>
__global__ void __launch_bounds__(32 * WARPS) rotate_rows_kernel(const RowsParams P) {
  __shared__ float2 tables[WARPS][MAX_HALF];
  constexpr int ROWS = 32 / G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const int64_t w = (int64_t)blockIdx.x * WARPS + warp;
  const int64_t token = w / P.share;
  if (token >= P.tokens) return;
  const Steps steps(ROWS, P.hq, P.hk, APPEND ? P.hk : 0);
  const int begin = (int)(w - token * P.share) * P.per_warp;
  const int end = begin + P.per_warp < steps.all() ? begin + P.per_warp : steps.all();
  const Lane L(P.R, lane % G, lane);
  const int row = lane / G;
  auto side_of = [&](int i, int& head) {
    const int side = i < steps.q ? 0 : i < steps.q + steps.k ? 1 : 2;
    head = (i - (side == 0 ? 0 : side == 1 ? steps.q : steps.q + steps.k)) * ROWS + row;
    return side;
  };
  auto fetch = [&](int i) {
    int head;
    const int side = side_of(i, head);
    const T* base = (const T*)(side == 0 ? P.Q : side == 1 ? P.K : P.V);
    const bool in = i < end && head < (side == 0 ? P.hq : P.hk) && L.e0 < P.R.D;
    return in ? load8<T>(base + token * P.ld + (int64_t)head * P.R.D + L.e0) : zero8<T>();
  };
  Raw<T> raw[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) raw[u] = fetch(begin + u);
  int pos;
  mst_paged::Slot slot = {true, 0};
  if (APPEND) {
    const int b = mst_paged::sequence_of(P.batch, (int)token, lane);
    if (b < 0) return;
    pos = mst_paged::position_of(P.batch, b, (int)token);
    if (pos < 0) return;
    slot = mst_paged::slot_of(P.cache, P.batch, b, pos, &g_bad_page);
  } else {
    pos = P.positions ? P.positions[token] : (int)(token % P.seq_len);
  }
  angles(tables[warp], P.R, pos, lane);
  const Turn turn = turn_of(P.R, L, tables[warp], false);
  float A[8], B[8];
  const float* gamma = nullptr;
  int cur = -1;
  for (int i0 = begin; i0 < end; i0 += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + u;
      if (i >= end) break;
      int head;
      const int side = side_of(i, head);
      if (side != cur && side < 2) {
        gamma = side == 0 ? P.R.gamma_q : P.R.gamma_k;
        weights(P.R, L, gamma, A, B);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          A[e] *= turn.c[e];
          B[e] *= turn.s[e];
        }
        cur = side;
      }
      Raw<T> out = raw[u];
      if (!APPEND || side < 2) {
        float x[8], p[8];
        widen(raw[u], x);
        partners(P.R, L, raw[u], x, p);
        float r = 1.f;
        if (gamma) {
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sq = fmaf(x[e], x[e], sq);
          r = rsqrtf(sum_lanes<G>(sq) / (float)P.R.D + P.R.eps);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r * fmaf(p[e], B[e], x[e] * A[e]);
        narrow(x, out);
      }
      if (head < (side == 0 ? P.hq : P.hk) && L.e0 < P.R.D) {
        if (side == 0 || !APPEND) {
          store8<T>((T*)(side == 0 ? P.Qo : P.Ko) + token * P.ldq + (int64_t)head * P.R.D + L.e0, out);
        } else if (slot.exists) {
          store8<T>((T*)(side == 1 ? P.cache.K : P.cache.V) + slot.at + (int64_t)head * P.cache.head_stride + L.e0, out);
        }
      }
    }
    if (i0 + AHEAD < end) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) raw[u] = fetch(i0 + AHEAD + u);
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ gradients
struct GradParams {
  Rotation R;
  const void *Q, *K, *dQo, *dKo;
  void *dQ, *dK;
  int64_t ld, lddo, ldg;
  int hq, hk;
  const int32_t* positions;
  int seq_len;
  int64_t tokens;
  int share, per_warp;
  float* partial;        // [blocks][2][D]: sums of the weights' gradients, or NULL
};

// Blocks that stay: each warp goes on to the token that lies a grid further, with its share of the weights' gradients in registers, so that a
// block leaves 2 D sums in all.
constexpr int GRAD_BLOCKS_PER_SM = 2, GRAD_AHEAD = 2;
constexpr int GRAD_BLOCKS_MOST = 512;

template <typename T, int G>
__global__ void __launch_bounds__(32 * WARPS, GRAD_BLOCKS_PER_SM) rotate_grad_kernel(const GradParams P) {
  __shared__ float2 tables[WARPS][MAX_HALF];
  constexpr int ROWS = 32 / G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const Steps steps(ROWS, P.hq, P.hk, 0);
  const Lane L(P.R, lane % G, lane);
  const int row = lane / G;
  const bool in_row = L.e0 < P.R.D;
  float acc[2][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[0][e] = acc[1][e] = 0.f;
  const int64_t all = P.tokens * P.share;
  for (int64_t w = (int64_t)blockIdx.x * WARPS + warp; w < all; w += (int64_t)gridDim.x * WARPS) {
    const int64_t token = w / P.share;
    const int begin = (int)(w - token * P.share) * P.per_warp;
    const int end = begin + P.per_warp < steps.all() ? begin + P.per_warp : steps.all();
    Raw<T> rx[GRAD_AHEAD], ry[GRAD_AHEAD];
    auto fetch = [&](int i, Raw<T>& x, Raw<T>& y) {
      const bool q = i < steps.q;
      const int head = (q ? i : i - steps.q) * ROWS + row;
      const bool in = i < end && head < (q ? P.hq : P.hk) && in_row;
      const int64_t at = (int64_t)head * P.R.D + L.e0;
      x = in && (q ? P.R.gamma_q : P.R.gamma_k) ? load8<T>((const T*)(q ? P.Q : P.K) + token * P.ld + at) : zero8<T>();
      y = in ? load8<T>((const T*)(q ? P.dQo : P.dKo) + token * P.lddo + at) : zero8<T>();
    };
#pragma unroll
    for (int u = 0; u < GRAD_AHEAD; ++u) fetch(begin + u, rx[u], ry[u]);
    angles(tables[warp], P.R, P.positions ? P.positions[token] : (int)(token % P.seq_len), lane);
    const Turn turn = turn_of(P.R, L, tables[warp], true);
    for (int i0 = begin; i0 < end; i0 += GRAD_AHEAD) {
      Raw<T> nx[GRAD_AHEAD], ny[GRAD_AHEAD];
      if (i0 + GRAD_AHEAD < end) {
#pragma unroll
        for (int u = 0; u < GRAD_AHEAD; ++u) fetch(i0 + GRAD_AHEAD + u, nx[u], ny[u]);
      }
#pragma unroll
      for (int u = 0; u < GRAD_AHEAD; ++u) {
        const int i = i0 + u;
        if (i >= end) break;
        const bool q = i < steps.q;
        const int head = (q ? i : i - steps.q) * ROWS + row;
        const float* gamma = q ? P.R.gamma_q : P.R.gamma_k;
        float y[8], z[8], p[8];
        widen(ry[u], y);
        partners(P.R, L, ry[u], y, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = fmaf(p[e], turn.s[e], y[e] * turn.c[e]);
        if (gamma) {
          float x[8], g[8], sq = 0.f, dot = 0.f;
          widen(rx[u], x);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = 0.f;
          if (in_row) {
            const float4 a = *reinterpret_cast<const float4*>(gamma + L.e0), b = *reinterpret_cast<const float4*>(gamma + L.e0 + 4);
            g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sq = fmaf(x[e], x[e], sq);
            dot = fmaf(z[e] * g[e], x[e], dot);
          }
          const float inv = 1.f / (float)P.R.D;
          const float r = rsqrtf(sum_lanes<G>(sq) * inv + P.R.eps);
          const float back = r * r * (sum_lanes<G>(dot) * inv);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float add = z[e] * x[e] * r;
            if (q) acc[0][e] += add; else acc[1][e] += add;
            z[e] = r * fmaf(-back, x[e], z[e] * g[e]);
          }
        }
        if (head < (q ? P.hq : P.hk) && in_row) {
          Raw<T> out;
          narrow(z, out);
          store8<T>((T*)(q ? P.dQ : P.dK) + token * P.ldg + (int64_t)head * P.R.D + L.e0, out);
        }
      }
#pragma unroll
      for (int u = 0; u < GRAD_AHEAD; ++u) {
        rx[u] = nx[u];
        ry[u] = ny[u];
      }
    }
  }
  if (!P.partial) return;
  // rows of a warp, then the warps, in a fixed order; the tables' place is free once every warp is here
  float* sums = reinterpret_cast<float*>(tables);   // [WARPS][G * 8]: 8 * 256 floats at most
  static_assert(sizeof(tables) >= sizeof(float) * WARPS * 256, "a block's sums fit the tables");
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = acc[side][e];
#pragma unroll
      for (int o = G; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane < G) sums[warp * (G * 8) + lane * 8 + e] = v;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < P.R.D; e += 32 * WARPS) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < WARPS; ++k) v += sums[k * (G * 8) + e];
      P.partial[((int64_t)blockIdx.x * 2 + side) * P.R.D + e] = v;
    }
  }
}

// the blocks' sums, in a fixed order: 32 columns a block, 32 rows of them at a time
__global__ void __launch_bounds__(1024) rotate_weight_grad_kernel(const float* partial, int blocks, int D, float* dgamma_q, float* dgamma_k) {
  __shared__ float part[32][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), first = threadIdx.x >> 5;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  float v = 0.f;
  if (c < 2 * D) {
#pragma unroll 4
    for (int b = first; b < blocks; b += 32) v += partial[(int64_t)b * 2 * D + c];
  }
  part[first][threadIdx.x & 31] = v;
  __syncthreads();
  if (first == 0 && c < 2 * D) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += part[k][threadIdx.x & 31];
    float* out = c < D ? dgamma_q : dgamma_k;
    if (out) out[c < D ? c : c - D] = s;
  }
}

// ------------------------------------------------------------------------------------------------------------ the calls
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

template <typename T, int G, bool APPEND>
mst_status_t launch_rows(RowsParams& P, cudaStream_t s) {
  const Steps steps(32 / G, P.hq, P.hk, APPEND ? P.hk : 0);
  P.share = warps_of_token(P.tokens, steps.all());
  P.per_warp = (steps.all() + P.share - 1) / P.share;
  P.share = (steps.all() + P.per_warp - 1) / P.per_warp;
  const int64_t blocks = (P.tokens * P.share + WARPS - 1) / WARPS;
  if (blocks > 0x7FFFFFFF) return MST_ERR_SHAPE;
  MST_CUDA_TRY(mst_launch_overlapped(rotate_rows_kernel<T, G, APPEND>, dim3((unsigned)blocks), dim3(32 * WARPS), 0, s, P));
  return MST_OK;
}
template <typename T, bool APPEND>
mst_status_t launch_rows(RowsParams& P, cudaStream_t s) {
  switch (lanes_of(P.R.D)) {
    case 1: return launch_rows<T, 1, APPEND>(P, s);
    case 2: return launch_rows<T, 2, APPEND>(P, s);
    case 4: return launch_rows<T, 4, APPEND>(P, s);
    case 8: return launch_rows<T, 8, APPEND>(P, s);
    case 16: return launch_rows<T, 16, APPEND>(P, s);
    default: return launch_rows<T, 32, APPEND>(P, s);
  }
}
template <typename T, int G>
mst_status_t launch_grad(GradParams& P, float* dgamma_q, float* dgamma_k, cudaStream_t s) {
  const Steps steps(32 / G, P.hq, P.hk, 0);
  P.share = warps_of_token(P.tokens, steps.all());
  P.per_warp = (steps.all() + P.share - 1) / P.share;
  P.share = (steps.all() + P.per_warp - 1) / P.per_warp;
  int64_t blocks = (P.tokens * P.share + WARPS - 1) / WARPS;
  const int64_t most = (int64_t)GRAD_BLOCKS_PER_SM * mst_sm_count();
  if (blocks > most) blocks = most;
  if (blocks > GRAD_BLOCKS_MOST) blocks = GRAD_BLOCKS_MOST;
  MST_CUDA_TRY(mst_launch_overlapped(rotate_grad_kernel<T, G>, dim3((unsigned)blocks), dim3(32 * WARPS), 0, s, P));
  if (P.partial)
    MST_CUDA_TRY(mst_launch_overlapped(rotate_weight_grad_kernel, dim3((unsigned)((2 * P.R.D + 31) / 32)), dim3(1024), 0, s,
                                       (const float*)P.partial, (int)blocks, P.R.D, dgamma_q, dgamma_k));
  return MST_OK;
}
template <typename T>
mst_status_t launch_grad(GradParams& P, float* dgamma_q, float* dgamma_k, cudaStream_t s) {
  switch (lanes_of(P.R.D)) {
    case 1: return launch_grad<T, 1>(P, dgamma_q, dgamma_k, s);
    case 2: return launch_grad<T, 2>(P, dgamma_q, dgamma_k, s);
    case 4: return launch_grad<T, 4>(P, dgamma_q, dgamma_k, s);
    case 8: return launch_grad<T, 8>(P, dgamma_q, dgamma_k, s);
    case 16: return launch_grad<T, 16>(P, dgamma_q, dgamma_k, s);
    default: return launch_grad<T, 32>(P, dgamma_q, dgamma_k, s);
  }
}

// counts and types that the training calls have in common
mst_status_t check_rows(mst_dtype_t dtype, int64_t tokens, int32_t seq_len, const int32_t* positions, int32_t hq, int32_t hk) {
  if (tokens < 0 || hq < 0 || hk < 0 || (!positions && seq_len <= 0)) return MST_ERR_INVALID_ARG;
  if (dtype != MST_F32 && dtype != MST_BF16) return MST_ERR_DTYPE;
  if (tokens > 0x7FFFFFFF || hq > 65535 || hk > 65535) return MST_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return MST_ERR_SHAPE;
  return MST_OK;
}
mst_status_t check_ld(int64_t ld, int32_t hq, int32_t hk, int D) {
  return ld % 8 != 0 || ld < (int64_t)hq * D || ld < (int64_t)hk * D ? MST_ERR_SHAPE : MST_OK;
}

}  // namespace

mst_status_t mst_append_error_flags(int32_t* flags) { return mst_paged::take_flag((const void*)&g_bad_page, flags); }

extern "C" mst_status_t mst_qk_norm_rotate_fwd(const mst_rotation_t* rotation, mst_dtype_t dtype, int64_t tokens, int32_t seq_len,
                                               const int32_t* positions, int32_t heads_q, int32_t heads_k, const void* Q,
                                               const void* K, int64_t ld, void* Q_out, void* K_out, int64_t ldo,
                                               mst_stream_t stream) {
  RowsParams P = {};
  MST_TRY(check(rotation, &P.R));
  MST_TRY(check_rows(dtype, tokens, seq_len, positions, heads_q, heads_k));
  if (heads_q == 0) Q = Q_out = nullptr;
  if (heads_k == 0) K = K_out = nullptr;
  if ((heads_q > 0 && (!Q || !Q_out)) || (heads_k > 0 && (!K || !K_out))) return MST_ERR_INVALID_ARG;
  MST_TRY(check_ld(ld, heads_q, heads_k, P.R.D));
  MST_TRY(check_ld(ldo, heads_q, heads_k, P.R.D));
  if (misaligned(Q) || misaligned(K) || misaligned(Q_out) || misaligned(K_out)) return MST_ERR_SHAPE;
  if (tokens == 0 || (heads_q == 0 && heads_k == 0)) return MST_OK;
  MST_TRY(mst_on_this_device({Q, K, Q_out, K_out, positions, P.R.inv_freq, P.R.gamma_q, P.R.gamma_k}));
  P.Q = Q; P.K = K; P.Qo = Q_out; P.Ko = K_out;
  P.ld = ld; P.ldq = ldo;
  P.hq = heads_q; P.hk = heads_k;
  P.positions = positions; P.seq_len = seq_len; P.tokens = tokens;
  return dtype == MST_BF16 ? launch_rows<__nv_bfloat16, false>(P, (cudaStream_t)stream) : launch_rows<float, false>(P, (cudaStream_t)stream);
}

extern "C" mst_status_t mst_qk_norm_rotate_bwd_workspace(const mst_rotation_t* rotation, int64_t tokens, size_t* bytes) {
  if (!bytes) return MST_ERR_INVALID_ARG;
  *bytes = 0;
  Rotation R;
  MST_TRY(check(rotation, &R));
  if (tokens < 0) return MST_ERR_INVALID_ARG;
  if (R.gamma_q || R.gamma_k) *bytes = sizeof(float) * GRAD_BLOCKS_MOST * 2 * (size_t)R.D;
  return MST_OK;
}

extern "C" mst_status_t mst_qk_norm_rotate_bwd(const mst_rotation_t* rotation, mst_dtype_t dtype, int64_t tokens, int32_t seq_len,
                                               const int32_t* positions, int32_t heads_q, int32_t heads_k, const void* Q,
                                               const void* K, int64_t ld, const void* dQ_out, const void* dK_out, int64_t lddo,
                                               void* dQ, void* dK, int64_t ldg, float* dgamma_q, float* dgamma_k, void* workspace,
                                               size_t workspace_bytes, mst_stream_t stream) {
  GradParams P = {};
  MST_TRY(check(rotation, &P.R));
  MST_TRY(check_rows(dtype, tokens, seq_len, positions, heads_q, heads_k));
  if (heads_q == 0) Q = dQ_out = dQ = nullptr;       // a side without heads has no pointers
  if (heads_k == 0) K = dK_out = dK = nullptr;
  if ((heads_q > 0 && (!dQ_out || !dQ || (P.R.gamma_q && !Q))) || (heads_k > 0 && (!dK_out || !dK || (P.R.gamma_k && !K))))
    return MST_ERR_INVALID_ARG;
  if ((dgamma_q && !P.R.gamma_q) || (dgamma_k && !P.R.gamma_k)) return MST_ERR_INVALID_ARG;
  MST_TRY(check_ld(ld, heads_q, heads_k, P.R.D));
  MST_TRY(check_ld(lddo, heads_q, heads_k, P.R.D));
  MST_TRY(check_ld(ldg, heads_q, heads_k, P.R.D));
  if (misaligned(Q) || misaligned(K) || misaligned(dQ_out) || misaligned(dK_out) || misaligned(dQ) || misaligned(dK) || misaligned(workspace) ||
      ((reinterpret_cast<uintptr_t>(dgamma_q) | reinterpret_cast<uintptr_t>(dgamma_k)) & 3u) != 0)
    return MST_ERR_SHAPE;
  const bool sums = dgamma_q || dgamma_k;
  if (sums) {
    size_t need = 0;
    MST_TRY(mst_qk_norm_rotate_bwd_workspace(rotation, tokens, &need));
    if (!workspace || workspace_bytes < need) return MST_ERR_CAPACITY;
  }
  const bool empty = tokens == 0 || (heads_q == 0 && heads_k == 0);
  if (empty && !sums) return MST_OK;
  MST_TRY(mst_on_this_device({Q, K, dQ_out, dK_out, dQ, dK, positions, P.R.inv_freq, P.R.gamma_q, P.R.gamma_k, dgamma_q, dgamma_k,
                              sums ? workspace : nullptr}));
  P.Q = Q; P.K = K;
  P.dQo = dQ_out; P.dKo = dK_out; P.dQ = dQ; P.dK = dK;
  P.ld = ld; P.lddo = lddo; P.ldg = ldg;
  P.hq = heads_q; P.hk = heads_k;
  P.positions = positions; P.seq_len = seq_len; P.tokens = tokens;
  P.partial = sums ? (float*)workspace : nullptr;
  if (empty) {   // sums over nothing
    if (dgamma_q) MST_CUDA_TRY(cudaMemsetAsync(dgamma_q, 0, sizeof(float) * P.R.D, (cudaStream_t)stream));
    if (dgamma_k) MST_CUDA_TRY(cudaMemsetAsync(dgamma_k, 0, sizeof(float) * P.R.D, (cudaStream_t)stream));
    return MST_OK;
  }
  return dtype == MST_BF16 ? launch_grad<__nv_bfloat16>(P, dgamma_q, dgamma_k, (cudaStream_t)stream)
                           : launch_grad<float>(P, dgamma_q, dgamma_k, (cudaStream_t)stream);
}

extern "C" mst_status_t mst_paged_append(const mst_paged_cache_t* cache, const mst_paged_batch_t* batch, const mst_rotation_t* rotation,
                                         int32_t heads_q, const void* Q, const void* K, const void* V, int64_t ld, void* Q_out,
                                         int64_t ldq, mst_stream_t stream) {
  RowsParams P = {};
  MST_TRY(mst_paged::check(cache, batch, &P.cache, &P.batch));
  if (rotation) {
    MST_TRY(check(rotation, &P.R));
    if (P.R.D != cache->head_dim) return MST_ERR_SHAPE;
  } else {
    P.R.D = cache->head_dim;
    if (P.R.D % 8 != 0 || P.R.D > 256) return MST_ERR_SHAPE;
  }
  if (!Q && !Q_out) heads_q = 0;
  if (heads_q == 0) Q = Q_out = nullptr;
  if (heads_q < 0 || !K || !V || (heads_q > 0 && (!Q || !Q_out))) return MST_ERR_INVALID_ARG;
  if (heads_q > 65535) return MST_ERR_SHAPE;
  MST_TRY(check_ld(ld, heads_q, cache->kv_heads, P.R.D));
  if (heads_q > 0) MST_TRY(check_ld(ldq, heads_q, 0, P.R.D));
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Q_out)) return MST_ERR_SHAPE;
  if (P.batch.batch == 0 || P.batch.tokens == 0) return MST_OK;
  MST_TRY(mst_on_this_device({Q, K, V, Q_out, P.R.inv_freq, P.R.gamma_q, P.R.gamma_k, P.cache.K, P.cache.V, P.batch.first, P.batch.len,
                              P.batch.table}));
  P.Q = Q; P.K = K; P.V = V; P.Qo = Q_out;
  P.ld = ld; P.ldq = ldq;
  P.hq = heads_q; P.hk = cache->kv_heads;
  P.tokens = P.batch.tokens;
  return launch_rows<__nv_bfloat16, true>(P, (cudaStream_t)stream);
}
