// Layer norm with weight and bias, forward and backward, for joint steps of blocks that carry it in RMSNorm's place:
//   mu = mean_i x_i,  r = 1 / sqrt(mean_i (x_i - mu)^2 + eps),  xh_i = (x_i - mu) r,  h_i = xh_i g_i + b_i
//   dx_i = r (g_i dh_i - mean_j (g_j dh_j) - xh_i mean_j (g_j dh_j xh_j)) + d_res_i,  dg_i = sum_t dh_i xh_i,  db_i = sum_t dh_i
// with dh = dh1 + dh2 + dh3.  HBM-bound: every tensor passes once.  A row is held in registers by a group of G lanes, C 16-byte
// chunks (8 values) a lane, so that the mean and the sum of squared distances from it are two reductions over registers (no
// cancellation of E x^2 - (E x)^2: a row may sit far from zero).  Arithmetic is float32.
#include <algorithm>

#include "faar_internal.h"

namespace faar {
namespace {

// A row's group: G lanes of a wavefront (8 .. 64, a workgroup of 256 threads holds 256 / G rows), or with kWide the whole workgroup
// of 2 to 16 wavefronts, one row at a time.
constexpr int kWide = 0;
constexpr int kMostD = 16384;          // entries of a row
template <int G> constexpr int rows_of() { return G == kWide ? 1 : 256 / (G == kWide ? 256 : G); }
template <int G> constexpr int most_threads() { return G == kWide ? 1024 : 256; }
template <int G> __device__ __forceinline__ int lanes_of() { return G == kWide ? blockDim.x : G; }

// sums of N values over a row's group, in every lane of it: by shuffles, and between wavefronts through LDS with one barrier (two sets
// of slots take turns: a set is written again only behind the barrier of the call after).  All threads of the workgroup call it together.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&a)[N], int turn) {
  constexpr int W = G == kWide ? 64 : G;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] += __shfl_xor(a[i], o);
  if constexpr (G == kWide) {
    __shared__ float part[2][N][16];
    const int w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) part[turn & 1][i][w] = a[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i] = 0.0f;
      for (int j = 0; j < nw; ++j) a[i] += part[turn & 1][i][j];
    }
  }
}

// 8 values as they lie in memory
template <typename XT> struct Raw8;
template <> struct Raw8<bf16_t> {
  uint4 q;
  __device__ __forceinline__ void load(const bf16_t* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t r[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    }
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};

// A workgroup's groups walk the rows with a stride and request the next row while they work on one; g and b stay in registers.
template <typename XT, int G, int C>
__global__ void __launch_bounds__(most_threads<G>())
k_layernorm_fwd(const XT* __restrict__ X, int64_t T, int D8, const float* __restrict__ g, const float* __restrict__ b, float eps,
                bf16_t* __restrict__ H, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int R = rows_of<G>();
  const int L = lanes_of<G>(), sub = threadIdx.x % L, grp = threadIdx.x / L;
  const float n = static_cast<float>(D8 * 8);
  Raw8<XT> next[C];
  auto request = [&](int64_t row) {
    if (row >= T) return;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (sub + c * L < D8) next[c].load(X + (row * D8 + sub + c * L) * 8);
  };
  request(blockIdx.x * (int64_t)R + grp);
  float gg[C][8], bb[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) gg[c][j] = bb[c][j] = 0.0f;
    if (sub + c * L < D8) {
      load8(g + (sub + c * L) * 8, gg[c]);
      if (b) load8(b + (sub + c * L) * 8, bb[c]);
    }
  }
  const int64_t stride = (int64_t)gridDim.x * R;
  for (int64_t row0 = blockIdx.x * (int64_t)R; row0 < T; row0 += stride) {
    const int64_t row = row0 + grp;
    const bool live = row < T;
    float x[C][8], s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!live || sub + c * L >= D8) continue;
      next[c].get(x[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0] += x[c][j];
    }
    request(row + stride);
    group_sum<G, 1>(s, 0);
    const float mu = s[0] / n;
    s[0] = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!live || sub + c * L >= D8) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[c][j] -= mu;
        s[0] = fmaf(x[c][j], x[c][j], s[0]);
      }
    }
    group_sum<G, 1>(s, 1);
    const float r = 1.0f / sqrtf(s[0] / n + eps);
    if (!live) continue;
    if (sub == 0) {
      mean[row] = mu;
      rstd[row] = r;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (sub + c * L >= D8) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[c][j] = fmaf(x[c][j] * r, gg[c][j], bb[c][j]);
      W8<bf16_t>::store(H + (row * D8 + sub + c * L) * 8, x[c]);
    }
  }
}

// A workgroup's groups walk the rows with a stride and request the next row while they work on one.  Where the weight's or the bias's
// gradient is wanted (kCols) each lane keeps the sums of its columns over its rows in registers, the groups of a workgroup add up
// through LDS, and the workgroups' partial sums [gridDim][2][D] are added by k_layernorm_cols in a fixed order.
// One chunk a lane and a row across several wavefronts, rather than a row a wavefront with four chunks a lane: a lane then has so few
// registers that the unit holds twice the wavefronts.  16384 rows of 2048, two dh and d_res, in us: a row a wavefront 90, a row on 4
// wavefronts 74 without the request ahead; rows of 5120 float32 on 4 wavefronts of 3 chunks a lane 63, on 8 of 2 46.
template <typename XT, int G, int C, bool kCols>
__global__ void __launch_bounds__(most_threads<G>())
k_layernorm_bwd(const bf16_t* __restrict__ dH1, const bf16_t* __restrict__ dH2, const bf16_t* __restrict__ dH3,
                const XT* __restrict__ X, int64_t T, int D8, const float* __restrict__ g, const float* __restrict__ mean,
                const float* __restrict__ rstd, const bf16_t* __restrict__ d_res, bf16_t* __restrict__ dX,
                float* __restrict__ partials) {
  constexpr int R = rows_of<G>();
  constexpr bool kAhead = C == 1;                      // two chunks a lane leave no registers for the next row, nor for g
  const int L = lanes_of<G>(), sub = threadIdx.x % L, grp = threadIdx.x / L;
  const float n = static_cast<float>(D8 * 8);
  // column sums: in registers, or with two chunks a lane (which would not fit there) each lane's own places in LDS
  constexpr bool kInLds = kCols && C > 1;
  float gg[C][8], dg[8], db[8];
  __shared__ __attribute__((aligned(16))) float sums[kInLds ? 2 * kMostD : 4];
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) gg[c][j] = 0.0f;
    if (kAhead && sub + c * L < D8) load8(g + (sub + c * L) * 8, gg[c]);
    if constexpr (kCols)
#pragma unroll
      for (int j = 0; j < 8; ++j) dg[j] = db[j] = 0.0f;
    if constexpr (kInLds)
      if (sub + c * L < D8) {
        store8(sums + (sub + c * L) * 8, dg);
        store8(sums + (D8 + sub + c * L) * 8, db);
      }
  }
  Raw8<XT> rx[C];
  Raw8<bf16_t> r1[C], r2[C], r3[C], rr[C];
  float mu_next = 0.0f, r_next = 0.0f;
  auto request = [&](int64_t row) {
    if (row >= T) return;
    mu_next = mean[row];
    r_next = rstd[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = sub + c * L;
      if (at >= D8) continue;
      const int64_t o = (row * D8 + at) * 8;
      rx[c].load(X + o);
      r1[c].load(dH1 + o);
      if (dH2) r2[c].load(dH2 + o);
      if (kAhead && dH3) r3[c].load(dH3 + o);
      if (kAhead && d_res) rr[c].load(d_res + o);
    }
  };
  const int64_t stride = (int64_t)gridDim.x * R;
  if constexpr (kAhead) request(blockIdx.x * (int64_t)R + grp);
  int turn = 0;
  for (int64_t row0 = blockIdx.x * (int64_t)R; row0 < T; row0 += stride) {
    const int64_t row = row0 + grp;
    const bool live = row < T;
    if constexpr (!kAhead) request(row);
    const float mu = mu_next, r = r_next;
    float xh[C][8], gd[C][8], res[8];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!live || sub + c * L >= D8) continue;
      float t[8];
      rx[c].get(xh[c]);
      r1[c].get(gd[c]);
      if (dH2) {
        r2[c].get(t);
#pragma unroll
        for (int j = 0; j < 8; ++j) gd[c][j] += t[j];
      }
      if (dH3) {
        if constexpr (kAhead) r3[c].get(t);
        else W8<bf16_t>::load(dH3 + (row * D8 + sub + c * L) * 8, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) gd[c][j] += t[j];
      }
      if constexpr (kAhead) {
#pragma unroll
        for (int j = 0; j < 8; ++j) res[j] = 0.0f;
        if (d_res) rr[c].get(res);
      } else {
        load8(g + (sub + c * L) * 8, gg[c]);
      }
      float* place = sums + (sub + c * L) * 8;
      if constexpr (kInLds) {
        load8(place, dg);
        load8(place + D8 * 8, db);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[c][j] = (xh[c][j] - mu) * r;
        if constexpr (kCols) {
          dg[j] = fmaf(gd[c][j], xh[c][j], dg[j]);
          db[j] += gd[c][j];
        }
        gd[c][j] *= gg[c][j];
        s[0] += gd[c][j];
        s[1] = fmaf(gd[c][j], xh[c][j], s[1]);
      }
      if constexpr (kInLds) {
        store8(place, dg);
        store8(place + D8 * 8, db);
      }
    }
    if constexpr (kAhead) request(row + stride);
    group_sum<G, 2>(s, turn++);
    const float m0 = s[0] / n, m1 = s[1] / n;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = sub + c * L;
      if (!live || at >= D8) continue;
      if constexpr (!kAhead) {
#pragma unroll
        for (int j = 0; j < 8; ++j) res[j] = 0.0f;
        if (d_res) W8<bf16_t>::load(d_res + (row * D8 + at) * 8, res);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) gd[c][j] = fmaf(r, fmaf(-xh[c][j], m1, gd[c][j] - m0), res[j]);
      W8<bf16_t>::store(dX + (row * D8 + at) * 8, gd[c]);
    }
  }
  if constexpr (kCols) {
    float* out = partials + blockIdx.x * (int64_t)2 * D8 * 8;
    if constexpr (R == 1) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int at = sub + c * L;
        if (at >= D8) continue;
        if constexpr (kInLds) {
          load8(sums + at * 8, dg);
          load8(sums + (D8 + at) * 8, db);
        }
        store8(out + at * 8, dg);
        store8(out + (D8 + at) * 8, db);
      }
    } else {
      // column sums of the groups: thread (grp, sub) leaves its 8 values of either, the first group adds up
      __shared__ float lds[256][9];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[threadIdx.x][j] = k ? db[j] : dg[j];
        __syncthreads();
        if (grp == 0 && sub < D8) {
          float a[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            a[j] = 0.0f;
            for (int q = 0; q < R; ++q) a[j] += lds[q * L + sub][j];
          }
          store8(out + ((int64_t)k * D8 + sub) * 8, a);
        }
      }
    }
  }
}

// dg, db = sums of the partial rows [P][2 D]: 16 columns of 4 values by 64 slices of the partial rows per workgroup
__global__ void __launch_bounds__(1024)
k_layernorm_cols(const float* __restrict__ partials, int P, int64_t D, float* __restrict__ dg, float* __restrict__ db) {
  const int col = threadIdx.x % 16, slice = threadIdx.x / 16;
  const int64_t at = (blockIdx.x * (int64_t)16 + col) * 4;         // of 2 D; D % 8 == 0: a run of 4 is all dg or all db
  __shared__ float4 part[64][16];
  float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (at < 2 * D) {
#pragma unroll 4
    for (int p = slice; p < P; p += 64) {
      const float4 v = *reinterpret_cast<const float4*>(partials + (int64_t)p * 2 * D + at);
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
  }
  part[slice][col] = a;
  __syncthreads();
#pragma unroll
  for (int half = 32; half > 0; half >>= 1) {          // the same order at every call
    if (slice < half) {
      const float4 v = part[slice + half][col];
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
      part[slice][col] = a;
    }
    __syncthreads();
  }
  float* out = at < D ? dg : db;
  if (slice == 0 && at < 2 * D && out) *reinterpret_cast<float4*>(out + (at < D ? at : at - D)) = a;
}

// threads of the workgroup that holds a row of D > 512 with one chunk (two, of D > 8192) a lane
int wide_threads(int64_t D) {
  const int64_t chunks = D / 8, per = D > 8192 ? 2 : 1;
  return static_cast<int>((chunks + 64 * per - 1) / (64 * per) * 64);
}
int group_of(int64_t D) { return D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : 64; }

}  // namespace

int64_t layernorm_partial_rows(int64_t T, int64_t D) {
  // workgroups of the backward, which walk the rows: 8 wavefronts a compute unit.  With the next row always on its way more only add
  // partial sums (16384 rows of 2048: 64 us with 8, 70 with 16; 89 with 4)
  const int threads = D <= 512 ? 256 : wide_threads(D), R = D <= 512 ? 256 / group_of(D) : 1;
  const int64_t most = 256 * std::max(1, 512 / threads), rows = (T + R - 1) / R;
  return std::min(rows, most);
}

// Forward: a row a wavefront up to 2048 entries (24 wavefronts a unit; 16384 rows of 2048: 27.6 us, against 28.8 with a row on four
// wavefronts, whose two barriers a row need all 32 a unit can hold to hide), a row a workgroup beyond (8192 rows of 4096: 28.4 us, a row
// a wavefront 49).
hipError_t launch_layernorm_fwd(const void* X, bool x_bf16, int64_t T, int64_t D, const float* g, const float* b, float eps, bf16_t* H,
                                float* mean, float* rstd, hipStream_t st) {
  const int d8 = static_cast<int>(D / 8);
#define FAAR_LN_F(GG, CC, NT, WAVES)                                                                                                    \
  do {                                                                                                                                 \
    const int nt = (NT);                                                                                                               \
    const int64_t R = rows_of<GG>();                                                                                                   \
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((T + R - 1) / R, 256 * std::max(1, (WAVES) * 64 / nt))));                  \
    if (x_bf16) hipLaunchKernelGGL((k_layernorm_fwd<bf16_t, GG, CC>), grid, dim3(nt), 0, st, static_cast<const bf16_t*>(X), T, d8, g, b, eps, H, mean, rstd); \
    else hipLaunchKernelGGL((k_layernorm_fwd<float, GG, CC>), grid, dim3(nt), 0, st, static_cast<const float*>(X), T, d8, g, b, eps, H, mean, rstd);           \
  } while (0)
  if (D <= 64) FAAR_LN_F(8, 1, 256, 24);
  else if (D <= 128) FAAR_LN_F(16, 1, 256, 24);
  else if (D <= 256) FAAR_LN_F(32, 1, 256, 24);
  else if (D <= 512) FAAR_LN_F(64, 1, 256, 24);
  else if (D <= 1024) FAAR_LN_F(64, 2, 256, 24);
  else if (D <= 2048) FAAR_LN_F(64, 4, 256, 24);
  else if (D <= 8192) FAAR_LN_F(kWide, 1, wide_threads(D), 32);
  else FAAR_LN_F(kWide, 2, wide_threads(D), 32);
#undef FAAR_LN_F
  return hipGetLastError();
}

hipError_t launch_layernorm_bwd(const bf16_t* dH1, const bf16_t* dH2, const bf16_t* dH3, const void* X, bool x_bf16, int64_t T, int64_t D,
                                const float* g, const float* mean, const float* rstd, const bf16_t* d_res, bf16_t* dX, float* dg,
                                float* db, float* partials, hipStream_t st) {
  const bool cols = dg || db;
  const int64_t P = layernorm_partial_rows(T, D);
  const dim3 grid(static_cast<unsigned>(P));
  const int d8 = static_cast<int>(D / 8);
#define FAAR_LN_B1(XT, GG, CC, NT, K) \
  hipLaunchKernelGGL((k_layernorm_bwd<XT, GG, CC, K>), grid, dim3(NT), 0, st, dH1, dH2, dH3, static_cast<const XT*>(X), T, d8, g, mean, rstd, d_res, dX, partials)
#define FAAR_LN_B(GG, CC, NT)                                                                                       \
  do {                                                                                                              \
    if (x_bf16) { if (cols) FAAR_LN_B1(bf16_t, GG, CC, NT, true); else FAAR_LN_B1(bf16_t, GG, CC, NT, false); }     \
    else        { if (cols) FAAR_LN_B1(float, GG, CC, NT, true); else FAAR_LN_B1(float, GG, CC, NT, false); }       \
  } while (0)
  if (D <= 64) FAAR_LN_B(8, 1, 256);
  else if (D <= 128) FAAR_LN_B(16, 1, 256);
  else if (D <= 256) FAAR_LN_B(32, 1, 256);
  else if (D <= 512) FAAR_LN_B(64, 1, 256);
  else if (D <= 8192) FAAR_LN_B(kWide, 1, wide_threads(D));
  else FAAR_LN_B(kWide, 2, wide_threads(D));
#undef FAAR_LN_B
#undef FAAR_LN_B1
  if (hipError_t e = hipGetLastError()) return e;
  if (cols)
    hipLaunchKernelGGL(k_layernorm_cols, dim3(static_cast<unsigned>((2 * D / 4 + 15) / 16)), dim3(1024), 0, st, partials, static_cast<int>(P), D, dg, db);
  return hipGetLastError();
}

}  // namespace faar
