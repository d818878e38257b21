// Rotary embedding over several position axes (time, height, width of a video's patches; a text token has the same position on
// every axis): frequency i of a head turns by the angle pos[axis[i]][t] freq[i].  With a, b the two entries that frequency i pairs
// ("rotate-half": i and i + rot / 2; neighbours: 2 i and 2 i + 1),
//   y_a = a cos - b sin,  y_b = b cos + a sin;     the inverse turns by the opposite angle and is the backward pass.
// Positions reach 2^31 and angles matter modulo a turn: the product position x frequency is taken in 64 bits, in turns, and only
// its fraction, at most half a turn, goes on in float32.
//
// HBM-bound (2 bytes in, 2 out an element), provided that the 64-bit products, the sine and the cosine are not taken per element:
// a workgroup makes those of its tokens once, into LDS, and applies them to all heads of q and k.  201 MB (16384 tokens, 16 + 8
// heads of 128) in 40 us, the rate of a large copy (31 us where a part of them is still in the chip's cache); 24 tokens take 2.6 us on the device.
#include "faar_internal.h"

namespace faar {
namespace {

// fraction of a turn in [-1/2, 1/2]
__device__ __forceinline__ float turn_of(int32_t pos, double turns_per_position) {
  const double t = static_cast<double>(pos) * turns_per_position;
  return static_cast<float>(t - rint(t));
}

template <int TB>
__global__ void __launch_bounds__(kEltThreads)
k_rope_axes(RopeTensor q, RopeTensor k, int64_t T, int dh, int half, const int32_t* __restrict__ pos, RopeAxes ax, float sign, bool pairs,
            bool copy_rest) {
  __shared__ __attribute__((aligned(16))) float cs[TB][2][kRopeMaxHalf];   // [token][cos, sin][frequency]
  const int64_t t0 = (blockIdx.y * (int64_t)gridDim.x + blockIdx.x) * TB;
  if (t0 >= T) return;
  const int nt = static_cast<int>(T - t0 < TB ? T - t0 : TB);
  for (int i = threadIdx.x; i < nt * half; i += kEltThreads) {
    const int t = i / half, f = i - t * half;
    const float turn = turn_of(pos[ax.axis[f] * T + t0 + t], ax.turns[f]);
    cs[t][0][f] = cospif(2.0f * turn);
    cs[t][1][f] = sign * sinpif(2.0f * turn);
  }
  __syncthreads();
  // units: token x head x run of 8 frequencies, then the chunks of 8 entries that are not rotated
  const int heads = q.heads + k.heads, runs = half / 8, rest = copy_rest ? (dh - 2 * half) / 8 : 0, per = runs + rest;
  for (int i = threadIdx.x; i < nt * heads * per; i += kEltThreads) {
    const int u = i % per, th = i / per, t = th / heads;
    int head = th - t * heads;
    const bool is_q = head < q.heads;
    const bf16_t* x = (is_q ? q.x : k.x) + (t0 + t) * (is_q ? q.ldx : k.ldx);
    bf16_t* y = (is_q ? q.y : k.y) + (t0 + t) * (is_q ? q.ldy : k.ldy);
    if (!is_q) head -= q.heads;
    x += head * dh;
    y += head * dh;
    if (u >= runs) {
      const int at = 2 * half + (u - runs) * 8;
      *reinterpret_cast<uint4*>(y + at) = *reinterpret_cast<const uint4*>(x + at);
      continue;
    }
    const int ia = pairs ? 16 * u : 8 * u, ib = pairs ? 16 * u + 8 : half + 8 * u;
    float a[8], b[8], c[8], s[8], ya[8], yb[8];
    W8<bf16_t>::load(x + ia, a);
    W8<bf16_t>::load(x + ib, b);
    load8(&cs[t][0][8 * u], c);
    load8(&cs[t][1][8 * u], s);
    if (pairs) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ya[2 * j] = a[2 * j] * c[j] - a[2 * j + 1] * s[j];
        ya[2 * j + 1] = a[2 * j + 1] * c[j] + a[2 * j] * s[j];
        yb[2 * j] = b[2 * j] * c[4 + j] - b[2 * j + 1] * s[4 + j];
        yb[2 * j + 1] = b[2 * j + 1] * c[4 + j] + b[2 * j] * s[4 + j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ya[j] = a[j] * c[j] - b[j] * s[j];
        yb[j] = b[j] * c[j] + a[j] * s[j];
      }
    }
    W8<bf16_t>::store(y + ia, ya);
    W8<bf16_t>::store(y + ib, yb);
  }
}

}  // namespace

hipError_t launch_rope_axes(const RopeTensor& q, const RopeTensor& k, int64_t T, int dh, int half, const int32_t* pos, const RopeAxes& ax,
                            bool inverse, bool pairs, bool copy_rest, hipStream_t st) {
  const float sign = inverse ? -1.0f : 1.0f;
  // four tokens a workgroup give each of its threads one sine at 64 frequencies; few tokens spread over the device one by one.  One / four
  // a workgroup, 16 + 8 heads of 128 and 8 + 8 of 64 taken together, in us: 64 tokens 3.6 / 4.5, 512 4.1 / 5.1, 2048 6.6 / 6.6,
  // 8192 18.0 / 15.4, 40000 97 / 87
  constexpr int64_t kRow = 1 << 23;                    // workgroups of a grid's row: a row has below 2^32 threads
  const int64_t n = (T + 3) / 4;
  if (T >= 2048)
    hipLaunchKernelGGL(k_rope_axes<4>, dim3(static_cast<unsigned>(n < kRow ? n : kRow), static_cast<unsigned>((n + kRow - 1) / kRow)), dim3(kEltThreads), 0, st, q, k, T, dh, half, pos, ax, sign, pairs, copy_rest);
  else
    hipLaunchKernelGGL(k_rope_axes<1>, dim3(static_cast<unsigned>(T)), dim3(kEltThreads), 0, st, q, k, T, dh, half, pos, ax, sign, pairs, copy_rest);
  return hipGetLastError();
}

}  // namespace faar
