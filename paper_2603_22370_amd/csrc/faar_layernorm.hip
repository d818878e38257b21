// Layer norm with weight and bias, forward and backward, for joint steps of blocks that carry it in RMSNorm's place:
//   mu = mean_i x_i,  r = 1 / sqrt(mean_i (x_i - mu)^2 + eps),  xh_i = (x_i - mu) r,  h_i = xh_i g_i + b_i
//   dx_i = r (g_i dh_i - mean_j (g_j dh_j) - xh_i mean_j (g_j dh_j xh_j)) + d_res_i,  dg_i = sum_t dh_i xh_i,  db_i = sum_t dh_i
// with dh = dh1 + dh2 + dh3.  HBM-bound: every tensor passes once.  A row is held in registers by a group of G lanes, C 16-byte
// chunks (8 values) a lane, so that the mean and the sum of squared distances from it are two reductions over registers (no
// cancellation of E x^2 - (E x)^2: a row may sit far from zero).  Arithmetic is float32.
#include "faar_internal.h"

namespace faar {
namespace {

// sums of N values over the G lanes of a row's group, in every lane of it; G up to 64 by shuffles, more through LDS.  All threads of
// the workgroup call it together.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&a)[N]) {
  constexpr int W = G < 64 ? G : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] += __shfl_xor(a[i], o);
  if constexpr (G > 64) {
    __shared__ float part[N][G / 64];
    __syncthreads();                                   // the previous use has been read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) part[i][threadIdx.x >> 6] = a[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < G / 64; ++w) a[i] += part[i][w];
    }
  }
}

template <int G> constexpr int threads_of() { return G < 256 ? 256 : G; }

template <typename XT, int G, int C>
__global__ void __launch_bounds__(threads_of<G>())
k_layernorm_fwd(const XT* __restrict__ X, int64_t T, int D8, const float* __restrict__ g, const float* __restrict__ b, float eps,
                bf16_t* __restrict__ H, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int R = threads_of<G>() / G;               // rows per workgroup
  const int sub = threadIdx.x % G;
  const int64_t row = blockIdx.x * (int64_t)R + threadIdx.x / G;
  const bool live = row < T;
  float x[C][8];
  float s[1] = {0.0f};
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = sub + c * G;
    if (live && at < D8) W8<XT>::load(X + (row * D8 + at) * 8, x[c]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) x[c][j] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s[0] += x[c][j];
  }
  group_sum<G, 1>(s);
  const float n = static_cast<float>(D8 * 8), mu = s[0] / n;
  s[0] = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (sub + c * G < D8)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[c][j] -= mu;
        s[0] += x[c][j] * x[c][j];
      }
  group_sum<G, 1>(s);
  const float r = 1.0f / sqrtf(s[0] / n + eps);
  if (!live) return;
  if (sub == 0) {
    mean[row] = mu;
    rstd[row] = r;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = sub + c * G;
    if (at >= D8) continue;
    float gg[8], bb[8];
    load8(g + at * 8, gg);
    if (b) load8(b + at * 8, bb);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) bb[j] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[c][j] = (x[c][j] * r) * gg[j] + bb[j];
    W8<bf16_t>::store(H + (row * D8 + at) * 8, x[c]);
  }
}

// A workgroup's groups walk the rows with a stride; where the weight's or the bias's gradient is wanted (kCols) each lane keeps the
// sums of its columns over its rows in registers, the groups of a workgroup add up through LDS, and the workgroups' partial sums
// [gridDim][2][D] are added by k_layernorm_cols in a fixed order.
template <typename XT, int G, int C, bool kCols>
__global__ void __launch_bounds__(threads_of<G>())
k_layernorm_bwd(const bf16_t* __restrict__ dH1, const bf16_t* __restrict__ dH2, const bf16_t* __restrict__ dH3,
                const XT* __restrict__ X, int64_t T, int D8, const float* __restrict__ g, const float* __restrict__ mean,
                const float* __restrict__ rstd, const bf16_t* __restrict__ d_res, bf16_t* __restrict__ dX,
                float* __restrict__ partials) {
  constexpr int NT = threads_of<G>(), R = NT / G;
  const int sub = threadIdx.x % G, grp = threadIdx.x / G;
  const float n = static_cast<float>(D8 * 8);
  float dg[kCols ? C : 1][8], db[kCols ? C : 1][8];
  if constexpr (kCols)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) dg[c][j] = db[c][j] = 0.0f;
  for (int64_t row0 = blockIdx.x * (int64_t)R; row0 < T; row0 += (int64_t)gridDim.x * R) {
    const int64_t row = row0 + grp;
    const bool live = row < T;
    const float mu = live ? mean[row] : 0.0f, r = live ? rstd[row] : 0.0f;
    float xh[C][8], gd[C][8];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = sub + c * G;
      const bool on = live && at < D8;
      const int64_t o = (row * D8 + at) * 8;
      if (on) {
        float t[8];
        W8<XT>::load(X + o, xh[c]);
        W8<bf16_t>::load(dH1 + o, gd[c]);
        if (dH2) {
          W8<bf16_t>::load(dH2 + o, t);
#pragma unroll
          for (int j = 0; j < 8; ++j) gd[c][j] += t[j];
        }
        if (dH3) {
          W8<bf16_t>::load(dH3 + o, t);
#pragma unroll
          for (int j = 0; j < 8; ++j) gd[c][j] += t[j];
        }
        load8(g + at * 8, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          xh[c][j] = (xh[c][j] - mu) * r;
          if constexpr (kCols) {
            dg[c][j] += gd[c][j] * xh[c][j];
            db[c][j] += gd[c][j];
          }
          gd[c][j] *= t[j];
          s[0] += gd[c][j];
          s[1] += gd[c][j] * xh[c][j];
        }
      }
    }
    group_sum<G, 2>(s);
    const float m0 = s[0] / n, m1 = s[1] / n;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = sub + c * G;
      if (!live || at >= D8) continue;
      const int64_t o = (row * D8 + at) * 8;
      float t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) gd[c][j] = r * (gd[c][j] - m0 - xh[c][j] * m1);
      if (d_res) {
        W8<bf16_t>::load(d_res + o, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) gd[c][j] += t[j];
      }
      W8<bf16_t>::store(dX + o, gd[c]);
    }
  }
  if constexpr (kCols) {
    float* out = partials + blockIdx.x * (int64_t)2 * D8 * 8;
    if constexpr (R == 1) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = sub + c * G;
        if (at >= D8) continue;
        store8(out + at * 8, dg[c]);
        store8(out + (D8 + at) * 8, db[c]);
      }
    } else {
      // column sums of the groups: one chunk index at a time, thread (grp, sub) leaves its 8 values, the first group adds up
      __shared__ float lds[NT][9];
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          __syncthreads();
#pragma unroll
          for (int j = 0; j < 8; ++j) lds[threadIdx.x][j] = k ? db[c][j] : dg[c][j];
          __syncthreads();
          const int at = sub + c * G;
          if (grp == 0 && at < D8) {
            float a[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              a[j] = 0.0f;
              for (int q = 0; q < R; ++q) a[j] += lds[q * G + sub][j];
            }
            store8(out + ((int64_t)k * D8 + at) * 8, a);
          }
        }
    }
  }
}

// dg, db = sums of the partial rows [P][2 D]: 16 columns of 4 values by 16 slices of the partial rows per workgroup
__global__ void __launch_bounds__(256)
k_layernorm_cols(const float* __restrict__ partials, int P, int64_t D, float* __restrict__ dg, float* __restrict__ db) {
  const int col = threadIdx.x % 16, slice = threadIdx.x / 16;
  const int64_t at = (blockIdx.x * (int64_t)16 + col) * 4;         // of 2 D; D % 8 == 0: a run of 4 is all dg or all db
  __shared__ float4 part[16][16];
  float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (at < 2 * D)
    for (int p = slice; p < P; p += 16) {
      const float4 v = *reinterpret_cast<const float4*>(partials + (int64_t)p * 2 * D + at);
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
  part[slice][col] = a;
  __syncthreads();
  if (slice != 0 || at >= 2 * D) return;
#pragma unroll
  for (int s = 1; s < 16; ++s) {
    const float4 v = part[s][col];
    a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
  }
  float* out = at < D ? dg : db;
  if (out) *reinterpret_cast<float4*>(out + (at < D ? at : at - D)) = a;
}

int groups_for(int64_t D) { return D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : D <= 2048 ? 64 : 256; }

}  // namespace

int64_t layernorm_partial_rows(int64_t T, int64_t D) {
  const int G = groups_for(D), R = (G < 256 ? 256 : G) / G;
  const int64_t rows = (T + R - 1) / R;
  return rows < 512 ? rows : 512;
}

// FN(group, chunks a lane): the group holds the row, with no more registers than it needs
#define FAAR_LN_DISPATCH(D, FN)                                                                          \
  do {                                                                                                   \
    if ((D) <= 64) FN(8, 1); else if ((D) <= 128) FN(16, 1); else if ((D) <= 256) FN(32, 1);             \
    else if ((D) <= 512) FN(64, 1); else if ((D) <= 1024) FN(64, 2); else if ((D) <= 2048) FN(64, 4);    \
    else if ((D) <= 4096) FN(256, 2); else if ((D) <= 8192) FN(256, 4); else FN(256, 8);                \
  } while (0)

hipError_t launch_layernorm_fwd(const void* X, bool x_bf16, int64_t T, int64_t D, const float* g, const float* b, float eps, bf16_t* H,
                                float* mean, float* rstd, hipStream_t st) {
  const int G = groups_for(D), NT = G < 256 ? 256 : G, R = NT / G;
  const dim3 grid(static_cast<unsigned>((T + R - 1) / R));
  const int d8 = static_cast<int>(D / 8);
#define FAAR_LN_F(GG, CC)                                                                                                              \
  do {                                                                                                                                 \
    if (x_bf16) hipLaunchKernelGGL((k_layernorm_fwd<bf16_t, GG, CC>), grid, dim3(NT), 0, st, static_cast<const bf16_t*>(X), T, d8, g, b, eps, H, mean, rstd); \
    else hipLaunchKernelGGL((k_layernorm_fwd<float, GG, CC>), grid, dim3(NT), 0, st, static_cast<const float*>(X), T, d8, g, b, eps, H, mean, rstd);           \
  } while (0)
  FAAR_LN_DISPATCH(D, FAAR_LN_F);
#undef FAAR_LN_F
  return hipGetLastError();
}

hipError_t launch_layernorm_bwd(const bf16_t* dH1, const bf16_t* dH2, const bf16_t* dH3, const void* X, bool x_bf16, int64_t T, int64_t D,
                                const float* g, const float* mean, const float* rstd, const bf16_t* d_res, bf16_t* dX, float* dg,
                                float* db, float* partials, hipStream_t st) {
  const int G = groups_for(D), NT = G < 256 ? 256 : G, R = NT / G;
  const bool cols = dg || db;
  const int64_t P = layernorm_partial_rows(T, D), rows = (T + R - 1) / R;
  const dim3 grid(static_cast<unsigned>(cols ? P : rows));
  const int d8 = static_cast<int>(D / 8);
#define FAAR_LN_B1(XT, GG, CC, K) \
  hipLaunchKernelGGL((k_layernorm_bwd<XT, GG, CC, K>), grid, dim3(NT), 0, st, dH1, dH2, dH3, static_cast<const XT*>(X), T, d8, g, mean, rstd, d_res, dX, partials)
#define FAAR_LN_B(GG, CC)                                                                  \
  do {                                                                                     \
    if (x_bf16) { if (cols) FAAR_LN_B1(bf16_t, GG, CC, true); else FAAR_LN_B1(bf16_t, GG, CC, false); } \
    else        { if (cols) FAAR_LN_B1(float, GG, CC, true); else FAAR_LN_B1(float, GG, CC, false); }   \
  } while (0)
  FAAR_LN_DISPATCH(D, FAAR_LN_B);
#undef FAAR_LN_B
#undef FAAR_LN_B1
  if (hipError_t e = hipGetLastError()) return e;
  if (cols)
    hipLaunchKernelGGL(k_layernorm_cols, dim3(static_cast<unsigned>((2 * D / 4 + 15) / 16)), dim3(256), 0, st, partials, static_cast<int>(P), D, dg, db);
  return hipGetLastError();
}

}  // namespace faar
