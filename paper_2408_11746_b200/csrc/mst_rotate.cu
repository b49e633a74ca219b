// Norm of queries and keys for each head with the position rotation in the same pass: forward, gradients, and the form that
// appends to a paged cache.  The arithmetic of a row is in mst_rotate.cuh; the kernels differ in where rows come from and go to.
//
// Each row is read once and written once.  A warp takes a token (or a share of its heads) and has the loads of its first steps in flight before it works
// out the angles; no block-wide step on the way.
// Bound: latency.  124 registers leave 16 warps an SM, each with three rows in flight, and a warp's instructions wait: forward (16384 tokens of 24 rows of
// 64, 24 us, 725 instructions a token) a quarter of the time for memory, a fifth for the instruction before, a tenth for shared memory, with issue slots 52 % busy
// and DRAM 29; gradients (40 rows, 56 us) a fifth for memory, a quarter for the instruction before, 57 % and 50.  Few tokens: a launch and a trip to memory.
#include "mst_paged.cuh"
#include "mst_rotate.cuh"

namespace {
using namespace mst_rot;

__device__ int g_bad_page = 0, g_bad_rows = 0;

struct RowsParams {
  Rotation R;
  const void *Q, *K, *V;
  void *Qo, *Ko;
  int64_t ld, ldq;
  int hq, hk;
  const int32_t* positions;
  int seq_len;
  int tokens;
  int groups_q, steps;         // groups of lanes that take queries, steps of a token's queries and keys
  int per_warp;                // steps of a warp, those of the values (appending) among them
  mst_paged::Cache cache;
  mst_paged::Batch batch;
};

template <typename T, int G, bool INTER, bool APPEND>
__global__ void __launch_bounds__(32 * WARPS, 2) rotate_rows_kernel(const __grid_constant__ RowsParams P) {
  constexpr int N = 4, AHEAD = sizeof(T) == 2 ? 3 : 2;      // steps whose loads are in flight together
  constexpr int ALL = 32 / G;
  __shared__ __align__(16) float2 tables[WARPS][MAX_HALF];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const unsigned at = blockIdx.x * WARPS + warp;
  if (at >= (unsigned)P.tokens) return;
  const int token = (int)at;
  const int begin = (int)blockIdx.y * P.per_warp, all_end = begin + P.per_warp;
  const int end = all_end < P.steps ? all_end : P.steps;
  const Lane L(P.R, lane % G, INTER, 2 * N);
  // this lane's side: its group's first head and how far apart its heads are
  const int group = lane / G;
  const bool is_q = group < P.groups_q;
  const int head0 = is_q ? group : group - P.groups_q, every = is_q ? P.groups_q : ALL - P.groups_q, heads = is_q ? P.hq : P.hk;
  const T* in = (const T*)(is_q ? P.Q : P.K) + token * P.ld + (int64_t)head0 * P.R.D;
  const int in_step = every * P.R.D;
  auto mine = [&](int i) { return i < end && L.in && head0 + i * every < heads; };
  Raw<T, N> raw[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    no_row(raw[u]);
    if (mine(begin + u)) load_row(raw[u], in + (int64_t)(begin + u) * in_step, L);
  }
  const float* gamma = is_q ? P.R.gamma_q : P.R.gamma_k;
  const Pairs<N> g = weights<INTER, N>(gamma, L);
  const Frequencies<G, N> F(P.R, lane);
  int pos;
  mst_paged::Slot slot = {true, 0};
  if (APPEND) {
    const int b = mst_paged::sequence_of(P.batch, token, lane, &g_bad_rows);
    if (b < 0) return;
    pos = mst_paged::position_of(P.batch, b, token);
    if (pos < 0) return;
    slot = mst_paged::slot_of(P.cache, P.batch, b, pos, &g_bad_page);
  } else {
    pos = P.positions ? P.positions[token] : (int)((unsigned)token % (unsigned)P.seq_len);
  }
  if (begin < P.steps) {
    const bool to_cache = APPEND && !is_q;
    T* out = to_cache ? (T*)P.cache.K + slot.at + head0 * P.cache.head_stride
                      : (T*)(is_q ? P.Qo : P.Ko) + token * P.ldq + (int64_t)head0 * P.R.D;
    const int64_t out_step = to_cache ? every * P.cache.head_stride : (int64_t)in_step;
    const bool writes = !to_cache || slot.exists;
    Pairs<N> A, B;      // what u (A) and v (B) are multiplied by: A.u, B.u for u', A.v, B.v for v'
    {
      const Turn<N> turn = turn_of<INTER>(tables[warp], P.R, Steps<G, N>(F), L, pos, lane);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        A.u[k] = mul2(g.u[k], turn.c[k]);
        A.v[k] = mul2(g.u[k], turn.s[k]);
        B.u[k] = negated(mul2(g.v[k], turn.s[k]));
        B.v[k] = mul2(g.v[k], turn.c[k]);
      }
    }
    const float inv_d = 1.f / (float)P.R.D;
    const bool norm = gamma != nullptr, alone = !L.turns;      // alone: no pairs, an infinite value stays on its own
    for (int i0 = begin; i0 < end; i0 += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u;
        if (i >= end) break;
        const Pairs<N> x = widen<INTER, N>(raw[u]);
        if (mine(i + AHEAD)) load_row(raw[u], in + (int64_t)(i + AHEAD) * in_step, L);
        Pairs<N> y;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          y.u[k] = mul2(x.u[k], A.u[k]);
          y.v[k] = mul2(x.v[k], B.v[k]);
        }
        if (!alone) {
#pragma unroll
          for (int k = 0; k < N; ++k) {
            y.u[k] = fma2(x.v[k], B.u[k], y.u[k]);
            y.v[k] = fma2(x.u[k], A.v[k], y.v[k]);
          }
        }
        const float sum = sum_lanes<G>(dot(x, x));       // every lane: it has shuffles
        const float r = norm ? rsqrtf(fmaf(sum, inv_d, P.R.eps)) : 1.f;
        const uint64_t r2 = pack2(r, r);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          y.u[k] = mul2(y.u[k], r2);
          y.v[k] = mul2(y.v[k], r2);
        }
        if (mine(i) && writes) {
          Raw<T, N> o;
          narrow<INTER, N>(y, o);
          store_row(o, out + i * out_step, L);
        }
      }
    }
  }
  if (APPEND && slot.exists) {      // the values are carried over as they are
    const int v0 = begin > P.steps ? begin - P.steps : 0, v1 = all_end - P.steps;
    const T* from = (const T*)P.V + token * P.ld;
    T* to = (T*)P.cache.V + slot.at;
    for (int i = v0; i < v1; ++i) {
      const int head = i * ALL + group;
      if (head < P.hk && L.in) {
        Raw<T, N> r;
        load_row(r, from + (int64_t)head * P.R.D, L);
        store_row(r, to + head * P.cache.head_stride, L);
      }
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
  int tokens;
  int groups_q, steps, share, per_warp;
  float* partial;        // [blocks][2][D]: sums of the weights' gradients, or NULL
};

// Blocks that stay: each warp goes on to the token that lies a grid further, with its share of the weights' gradients in registers, so that a
// block leaves 2 D sums in all.
constexpr int GRAD_BLOCKS_PER_SM = 2;
constexpr int GRAD_BLOCKS_MOST = 512;

template <typename T, int G, int N, bool INTER>
__global__ void __launch_bounds__(32 * WARPS, GRAD_BLOCKS_PER_SM) rotate_grad_kernel(const __grid_constant__ GradParams P) {
  constexpr int ALL = 32 / G, AHEAD = sizeof(T) * N <= 4 ? 3 : 1;
  __shared__ __align__(16) float2 tables[WARPS][MAX_HALF];
  __shared__ float sums[WARPS][2][256];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mst_grid_launch_dependents();
  mst_grid_dependency_wait();
  const Lane L(P.R, lane % G, INTER, 2 * N);
  const int group = lane / G;
  const bool is_q = group < P.groups_q;
  const int head0 = is_q ? group : group - P.groups_q, every = is_q ? P.groups_q : ALL - P.groups_q, heads = is_q ? P.hq : P.hk;
  const int step = every * P.R.D;
  const float* gamma = is_q ? P.R.gamma_q : P.R.gamma_k;
  const bool norm = gamma != nullptr, alone = !L.turns;
  const float inv_d = 1.f / (float)P.R.D;
  const Pairs<N> g = weights<INTER, N>(gamma, L);
  const Steps<G, N> steps{Frequencies<G, N>(P.R, lane)};
  Pairs<N> acc = {};
  const unsigned groups = ((unsigned)P.tokens + WARPS - 1) / WARPS, all = groups * (unsigned)P.share;
  for (unsigned unit = blockIdx.x; unit < all; unit += gridDim.x) {
    const unsigned part = P.share > 1 ? unit / groups : 0u, at = (unit - part * groups) * WARPS + warp;
    if (at >= (unsigned)P.tokens) continue;
    const int token = (int)at;
    const int begin = (int)part * P.per_warp;
    const int end = begin + P.per_warp < P.steps ? begin + P.per_warp : P.steps;
    const int64_t off = (int64_t)head0 * P.R.D;
    const T* x_in = (const T*)(is_q ? P.Q : P.K) + token * P.ld + off;
    const T* y_in = (const T*)(is_q ? P.dQo : P.dKo) + token * P.lddo + off;
    T* out = (T*)(is_q ? P.dQ : P.dK) + token * P.ldg + off;
    auto mine = [&](int i) { return i < end && L.in && head0 + i * every < heads; };
    Raw<T, N> rx[AHEAD], ry[AHEAD];
    auto fetch = [&](int i, Raw<T, N>& x, Raw<T, N>& y) {
      if (mine(i)) {
        load_row(y, y_in + (int64_t)i * step, L);
        if (norm) load_row(x, x_in + (int64_t)i * step, L);
      }
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      no_row(rx[u]);
      no_row(ry[u]);
      fetch(begin + u, rx[u], ry[u]);
    }
    const Turn<N> turn = turn_of<INTER>(tables[warp], P.R, steps, L, P.positions ? P.positions[token] : (int)((unsigned)token % (unsigned)P.seq_len), lane);
    for (int i0 = begin; i0 < end; i0 += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u;
        if (i >= end) break;
        const bool here = mine(i);
        const Pairs<N> y = widen<INTER, N>(ry[u]), x = widen<INTER, N>(rx[u]);
        fetch(i + AHEAD, rx[u], ry[u]);
        Pairs<N> z;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          z.u[k] = mul2(y.u[k], turn.c[k]);
          z.v[k] = mul2(y.v[k], turn.c[k]);
        }
        if (!alone) {
#pragma unroll
          for (int k = 0; k < N; ++k) {
            z.u[k] = fma2(y.v[k], turn.s[k], z.u[k]);
            z.v[k] = fma2(y.u[k], negated(turn.s[k]), z.v[k]);
          }
        }
        Pairs<N> zg;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          zg.u[k] = mul2(z.u[k], g.u[k]);
          zg.v[k] = mul2(z.v[k], g.v[k]);
        }
        const float sq = sum_lanes<G>(dot(x, x)), sd = sum_lanes<G>(dot(zg, x));     // every lane: they have shuffles
        if (norm) {
          const float r = rsqrtf(fmaf(sq, inv_d, P.R.eps)), back = -r * r * (sd * inv_d);
          const uint64_t r2 = pack2(r, r), b2 = pack2(back, back);
#pragma unroll
          for (int k = 0; k < N; ++k) {
            if (here) {       // rows that are not there may be another step's
              acc.u[k] = fma2(z.u[k], mul2(x.u[k], r2), acc.u[k]);
              acc.v[k] = fma2(z.v[k], mul2(x.v[k], r2), acc.v[k]);
            }
            z.u[k] = mul2(r2, fma2(b2, x.u[k], zg.u[k]));
            z.v[k] = mul2(r2, fma2(b2, x.v[k], zg.v[k]));
          }
        }
        if (here) {
          Raw<T, N> o;
          narrow<INTER, N>(z, o);
          store_row(o, out + (int64_t)i * step, L);
        }
      }
    }
  }
  if (!P.partial) return;
  // the groups of a warp, then the warps, in a fixed order
  for (int e = threadIdx.x; e < WARPS * 2 * 256; e += 32 * WARPS) (&sums[0][0][0])[e] = 0.f;
  __syncthreads();
  float v[4 * N];
  values_of<INTER, N>(acc, v);
  float* to = sums[warp][is_q ? 0 : 1];
#pragma unroll 1
  for (int k = 0; k < ALL; ++k) {
    if (group == k && L.in) {
#pragma unroll
      for (int e = 0; e < 2 * N; ++e) {
        to[L.near + e] += v[e];
        if (L.in_far) to[L.far + e] += v[2 * N + e];
      }
    }
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * P.R.D; e += 32 * WARPS) {
    const int side = e >= P.R.D, i = e - side * P.R.D;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) t += sums[k][side][i];
    P.partial[((int64_t)blockIdx.x * 2 + side) * P.R.D + i] = t;
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

template <typename T, int G, bool INTER, bool APPEND>
mst_status_t launch_rows(RowsParams& P, cudaStream_t s) {
  const Groups g = groups_of(G, P.hq, P.hk);
  P.groups_q = g.q;
  P.steps = g.steps;
  const int share = share_token(P.tokens, g.steps + (APPEND ? (P.hk + 32 / G - 1) / (32 / G) : 0), &P.per_warp);
  const unsigned blocks = ((unsigned)P.tokens + WARPS - 1) / WARPS;
  if (share > 65535) return MST_ERR_SHAPE;
  MST_CUDA_TRY(mst_launch_overlapped(rotate_rows_kernel<T, G, INTER, APPEND>, dim3(blocks, (unsigned)share), dim3(32 * WARPS), 0, s, P));
  return MST_OK;
}
template <typename T, bool INTER, bool APPEND>
mst_status_t launch_rows(RowsParams& P, cudaStream_t s) {
  switch (lanes_of(P.R.D, 4)) {
    case 2: return launch_rows<T, 2, INTER, APPEND>(P, s);
    case 4: return launch_rows<T, 4, INTER, APPEND>(P, s);
    case 8: return launch_rows<T, 8, INTER, APPEND>(P, s);
    default: return launch_rows<T, 16, INTER, APPEND>(P, s);
  }
}
template <typename T, bool APPEND>
mst_status_t launch_rows(RowsParams& P, cudaStream_t s) {
  return P.R.inter ? launch_rows<T, true, APPEND>(P, s) : launch_rows<T, false, APPEND>(P, s);
}
template <typename T, int G, int N, bool INTER>
mst_status_t launch_grad(GradParams& P, float* dgamma_q, float* dgamma_k, cudaStream_t s) {
  const Groups g = groups_of(G, P.hq, P.hk);
  P.groups_q = g.q;
  P.steps = g.steps;
  P.share = share_token(P.tokens, g.steps, &P.per_warp);
  int64_t blocks = ((int64_t)P.tokens + WARPS - 1) / WARPS * P.share;
  const int64_t most = (int64_t)GRAD_BLOCKS_PER_SM * mst_sm_count();
  if (blocks > most) blocks = most;
  if (blocks > GRAD_BLOCKS_MOST) blocks = GRAD_BLOCKS_MOST;
  MST_CUDA_TRY(mst_launch_overlapped(rotate_grad_kernel<T, G, N, INTER>, dim3((unsigned)blocks), dim3(32 * WARPS), 0, s, P));
  if (P.partial)
    MST_CUDA_TRY(mst_launch_overlapped(rotate_weight_grad_kernel, dim3((unsigned)((2 * P.R.D + 31) / 32)), dim3(1024), 0, s,
                                       (const float*)P.partial, (int)blocks, P.R.D, dgamma_q, dgamma_k));
  return MST_OK;
}
template <typename T, bool INTER>
mst_status_t launch_grad(GradParams& P, float* dgamma_q, float* dgamma_k, cudaStream_t s) {
  switch (lanes_of(P.R.D, 2)) {
    case 4: return launch_grad<T, 4, 2, INTER>(P, dgamma_q, dgamma_k, s);
    case 8: return launch_grad<T, 8, 2, INTER>(P, dgamma_q, dgamma_k, s);
    case 16: return launch_grad<T, 16, 2, INTER>(P, dgamma_q, dgamma_k, s);
    default: return launch_grad<T, 16, 4, INTER>(P, dgamma_q, dgamma_k, s);      // two groups in a warp at least: one for each side
  }
}
template <typename T>
mst_status_t launch_grad(GradParams& P, float* dgamma_q, float* dgamma_k, cudaStream_t s) {
  return P.R.inter ? launch_grad<T, true>(P, dgamma_q, dgamma_k, s) : launch_grad<T, false>(P, dgamma_q, dgamma_k, s);
}

// counts and types that the training calls have in common
mst_status_t check_rows(mst_dtype_t dtype, int64_t tokens, int32_t seq_len, const int32_t* positions, int32_t hq, int32_t hk) {
  if (tokens < 0 || hq < 0 || hk < 0 || (tokens > 0 && !positions && seq_len <= 0)) return MST_ERR_INVALID_ARG;
  if (dtype != MST_F32 && dtype != MST_BF16) return MST_ERR_DTYPE;
  if (tokens > 0x7FFFFFFF || hq > 65535 || hk > 65535) return MST_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return MST_ERR_SHAPE;
  return MST_OK;
}
mst_status_t check_ld(int64_t ld, int32_t hq, int32_t hk, int D) {
  return ld % 8 != 0 || ld < (int64_t)hq * D || ld < (int64_t)hk * D ? MST_ERR_SHAPE : MST_OK;
}

}  // namespace

mst_status_t mst_append_error_flags(int32_t* flags) {
  int32_t pages = 0, rows = 0;
  MST_TRY(mst_paged::take_flag((const void*)&g_bad_page, &pages));
  MST_TRY(mst_paged::take_flag((const void*)&g_bad_rows, &rows));
  *flags = pages | (rows << 2);
  return MST_OK;
}

extern "C" mst_status_t mst_qk_norm_rotate_fwd(const mst_rotation_t* rotation, mst_dtype_t dtype, int64_t tokens, int32_t seq_len,
                                               const int32_t* positions, int32_t heads_q, int32_t heads_k, const void* Q,
                                               const void* K, int64_t ld, void* Q_out, void* K_out, int64_t ldo,
                                               mst_stream_t stream) {
  RowsParams P = {};
  MST_TRY(check(rotation, &P.R));
  MST_TRY(check_rows(dtype, tokens, seq_len, positions, heads_q, heads_k));
  if (heads_q == 0) Q = Q_out = nullptr;
  if (heads_k == 0) K = K_out = nullptr;
  if (tokens > 0 && ((heads_q > 0 && (!Q || !Q_out)) || (heads_k > 0 && (!K || !K_out)))) return MST_ERR_INVALID_ARG;
  MST_TRY(check_ld(ld, heads_q, heads_k, P.R.D));
  MST_TRY(check_ld(ldo, heads_q, heads_k, P.R.D));
  if (misaligned(Q) || misaligned(K) || misaligned(Q_out) || misaligned(K_out)) return MST_ERR_SHAPE;
  if (tokens == 0 || (heads_q == 0 && heads_k == 0)) return MST_OK;
  MST_TRY(mst_on_this_device({Q, K, Q_out, K_out, positions, P.R.inv_freq, P.R.gamma_q, P.R.gamma_k}));
  P.Q = Q; P.K = K; P.Qo = Q_out; P.Ko = K_out;
  P.ld = ld; P.ldq = ldo;
  P.hq = heads_q; P.hk = heads_k;
  P.positions = positions; P.seq_len = seq_len; P.tokens = (int)tokens;
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
  if (tokens > 0 && ((heads_q > 0 && (!dQ_out || !dQ || (P.R.gamma_q && !Q))) || (heads_k > 0 && (!dK_out || !dK || (P.R.gamma_k && !K)))))
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
  P.positions = positions; P.seq_len = seq_len; P.tokens = (int)tokens;
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
  if (heads_q < 0 || (P.batch.tokens > 0 && (!K || !V || (heads_q > 0 && (!Q || !Q_out))))) return MST_ERR_INVALID_ARG;
  if (heads_q > 65535) return MST_ERR_SHAPE;
  MST_TRY(check_ld(ld, heads_q, cache->kv_heads, P.R.D));
  if (heads_q > 0) MST_TRY(check_ld(ldq, heads_q, 0, P.R.D));
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Q_out)) return MST_ERR_SHAPE;
  if (P.batch.batch == 0 || P.batch.tokens == 0) return MST_OK;
  if (cache->K == cache->V) return MST_ERR_INVALID_ARG;      // a row's key and value would be written to one place
  MST_TRY(mst_on_this_device({Q, K, V, Q_out, P.R.inv_freq, P.R.gamma_q, P.R.gamma_k, P.cache.K, P.cache.V, P.batch.first, P.batch.len,
                              P.batch.table}));
  P.Q = Q; P.K = K; P.V = V; P.Qo = Q_out;
  P.ld = ld; P.ldq = ldq;
  P.hq = heads_q; P.hk = cache->kv_heads;
  P.tokens = P.batch.tokens;
  return launch_rows<__nv_bfloat16, true>(P, (cudaStream_t)stream);
}
