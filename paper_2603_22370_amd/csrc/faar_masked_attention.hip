// Attention between the q / k / v and the output projections of blocks whose scores are capped by a tanh or carry a bias that falls
// with the distance, under document, prefix, window and whole-sequence masks; forward and backward over ragged sequences, and the
// forward for one token a sequence over a cache.  For a query at position p of its sequence and a key at position j, both of one
// head and key / value head,
//   z = scale q.k,  s = cap tanh(z / cap) - slope |p - j|  (no cap: z),  P = softmax of s over the keys that p sees,  o = P v
//   dv = P^T dO,  ds = P (dO v^T - rowsum(dO o)),  dz = ds (1 - tanh^2),  dq = scale dz k,  dk = scale dz^T q.
//
// Masks.  With the queries as the last positions of their sequence, what the masks leave of a query's keys is an interval
// [lo(p), hi(p)) whose ends grow with p, and so are the queries that see a key.  A block of 64 keys is then skipped, taken whole, or
// compared element by element (one subtraction, one comparison), and blocks outside a tile's interval are never loaded.
//
// Plan.  Sequence lengths live on the device.  A plan, made by one small launch for a batch and read by every layer, lists the work
// items: tiles of 128 queries (forward, dq) and of 64 keys (dk, dv) that each lie inside one sequence, the most expensive first, or
// for single tokens the pieces of the caches.  A workgroup reads its item with one load; the grid is the largest number of
// items that any lengths can give, and workgroups behind the last item end at once.
//
// Tiles, copies and products are those of the causal kernels (faar_attention.hip): 64-token tiles in LDS by asynchronous copies, two
// stages, 32 queries (keys) a wavefront, v_mfma_f32_32x32x16_bf16, probabilities in the accumulator layout as the next operand.
// P and dz are rounded to bf16 as matrix-core operands, like there: exact ones would be a second product each, and the outputs are
// bf16.  Everything else is float32, and what a rounding would do where a softmax is sharp is kept out of it: there dP - rowsum(dO o)
// is a small difference of large numbers, and rowsum has to be the mean of dP under P to more than the digits of bf16.
//   * o is divided by the sum of the ROUNDED probabilities (lse keeps that of the others): its error is then sum P eps (v - o) instead of
//     sum P eps v, as small as the difference itself.  A dot product of two pairs adds two rounded probabilities per instruction.
//   * next to o the forward can leave the 8 bits that follow each of its bf16 values (o_low), and the backward takes o to 16 significant bits.
// Norm-wise error of dq against 64 bits on 13 sequences whose scores have a deviation of 9 (10007 queries, 16 heads of 80): without the two
// 7.4e-3, with them 3.3e-3 (a third of it the output's own rounding, a third that of dz).
#include <algorithm>

#include "faar_attention_tile.h"

namespace faar {
namespace {

constexpr float kLowest = -1.7e38f;    // "no score yet": below every score, and finite, so that differences stay numbers
constexpr float kLazy = 8.0f;          // the reference maximum is raised when a score exceeds it by more than 2^kLazy

// how scores become exponents: as they are; with a bias; capped with every exponent in range of a fixed reference; capped with a
// running maximum (and a bias); the same under a wide cap
enum { kPlain = 0, kBiased = 1, kBounded = 2, kCapped = 3, kWide = 4 };
// how the backward undoes it
enum { kNoCap = 0, kNarrowCap = 1, kWideCap = 2 };

__device__ __attribute__((aligned(16))) const uint32_t kZeroChunk[4] = {0, 0, 0, 0};

// 16 bytes per lane from that lane's own address
__device__ __forceinline__ void dma16_from(const void* gptr, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(gptr) : "memory", "m0");
}
// What a head's width asks of the tiles: DH entries a row in LDS, KS steps of 16 in products over dh, DT blocks of 32 in products that give dh
struct Heads64 { static constexpr int DH = 64, KS = 4, DT = 2; };
struct Heads96 { static constexpr int DH = 128, KS = 6, DT = 3; };    // a row as of 128, of which the last quarter is never touched
struct Heads128 { static constexpr int DH = 128, KS = 8, DT = 4; };
// Products over dh leave out the last step where no head reaches it (13 images of 10007 patches, heads of 80: forward 121.6 -> 120.3 us,
// dq 150.9 -> 146.3, dk and dv 222.3 -> 219.4; not with 128, whose dk and dv have no register left for it)
template <class H> __device__ __forceinline__ bool uses_last(int dh) { return H::KS == 8 || dh > 16 * (H::KS - 1); }

// 64 rows of a tile of which `valid` are there, dh columns of each.  Columns beyond dh are left alone (clear_columns); rows that are
// missing are filled with zeros (a masked probability of 0 times whatever lies behind a sequence would not be 0 for all values).
template <int DH>
__device__ __forceinline__ void copy_tile(const bf16_t* __restrict__ src, int64_t row0, int valid, int64_t ld, int64_t col0, int dh,
                                          uint32_t lane_offset, uint32_t tile, int wave, int tid) {
  typedef Tile<DH> Tl;
  // the address of the tile, the same for all lanes, in scalar registers: said lane by lane, where the compiler does not see it
  const uint64_t at = reinterpret_cast<uint64_t>(src + row0 * ld + col0);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
  const bf16_t* base = reinterpret_cast<const bf16_t*>(static_cast<uint64_t>(hi) << 32 | lo);
  if (valid >= kTok && dh == DH) {
    Tl::copy(base, 0, kTok, ld, 0, lane_offset, tile, wave);
    return;
  }
  asm volatile("" : "+v"(tid));        // lanes' own addresses are formed here, where few blocks come by, and not kept in registers throughout
  const int r = tid / Tl::CPR, col = ((tid % Tl::CPR) ^ Tl::key(r)) * 8;
  if (col >= dh) return;               // these lanes copy nothing
  if (valid >= kTok) {
    Tl::copy(base, 0, kTok, ld, 0, lane_offset, tile, wave);
    return;
  }
#pragma unroll
  for (int j = 0; j < Tl::COPIES; ++j) {
    const int row = r + j * (256 / Tl::CPR);
    const void* p = row < valid ? static_cast<const void*>(src + (row0 + row) * ld + col0 + col) : kZeroChunk;
    dma16_from(p, __builtin_amdgcn_readfirstlane(tile + 4096u * j + 1024u * wave));
  }
}
// zeros in the columns from dh on that the products read, of `tiles` tiles: once a workgroup, since no copy touches them
template <class H>
__device__ __forceinline__ void clear_columns(bf16_t* tile, int tiles, int dh, int tid) {
  typedef Tile<H::DH> Tl;
  if (dh >= 16 * H::KS) return;
  const int r = tid / Tl::CPR, c = tid % Tl::CPR, col = (c ^ Tl::key(r)) * 8;
  if (col < dh || col >= 16 * H::KS) return;
  for (int i = 0; i < tiles; ++i)
    for (int j = 0; j < Tl::COPIES; ++j)
      *reinterpret_cast<uint4*>(tile + i * Tl::ELEMS + (r + j * (256 / Tl::CPR)) * H::DH + c * 8) = make_uint4(0, 0, 0, 0);
}

struct Seen { int lo, hi; };           // keys [lo, hi) of the sequence; hi <= lo: none
__device__ __forceinline__ Seen keys_of(int p, int k_len, int prefix, int window, bool causal) {
  int lo = 0, hi = causal ? max(p + 1, prefix) : k_len;
  if (window > 0) {
    lo = max(lo, p - window + 1);
    hi = min(hi, p + window);
  }
  return {lo, min(hi, k_len)};
}
// queries [lo, hi) of the sequence (by index, query i at position i + off) that see key j
__device__ __forceinline__ Seen queries_of(int j, int q_len, int off, int prefix, int window, bool causal) {
  int lo = 0, hi = q_len;
  if (causal && j >= prefix) lo = max(lo, j - off);
  if (window > 0) {
    lo = max(lo, j - off - window + 1);                // in this order: j - off is at most q_len
    hi = min(hi, j - off + window);
  }
  return {lo, hi};
}

// ---- the plan -----------------------------------------------------------------------------------------------------------------
constexpr int kSmallCaches = 4 * kPieceKeys;   // single tokens: rows of all caches
constexpr int kJoinThreads = 1024;     // a workgroup that adds up pieces
constexpr int kPlanThreads = 1024, kBuckets = 128, kLeastPiece = 8;

__device__ __forceinline__ bool inside(int start, int len, int T) { return start >= 0 && len >= 0 && start <= T && len <= T - start; }

// One workgroup: three passes over the tiles of all sequences, whose counts meet in LDS (or, for single tokens, one scan over the
// sequences).  Latency: 5-6 us for tens of sequences, 17 for one of 8192 tokens, once for all layers.
__global__ void __launch_bounds__(kPlanThreads)
k_attention_plan(const int* __restrict__ q_start, const int* __restrict__ q_len, const int* __restrict__ k_start, const int* __restrict__ k_len,
                 const int* __restrict__ prefix, PlanTag tag, PlanSizes z, int* __restrict__ plan) {
  const int n_seq = tag.w[kTagSeqs], Tq = tag.w[kTagTq], Tk = tag.w[kTagTk], window = tag.w[kTagWindow];
  const bool causal = tag.w[kTagFlags] & 1, single = tag.w[kTagFlags] & 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ unsigned long long sums[2];              // rows of q, of k
  __shared__ unsigned long long total[2];
  __shared__ float per_cost[2];
  __shared__ int longest[2], most_of_piece[2], slots[2], joins[2], unordered[2], shared_rows[2], bad, hist[2][kBuckets], scan[kPlanThreads], carry;
  if (tid < 2) {
    sums[tid] = total[tid] = 0;
    longest[tid] = slots[tid] = joins[tid] = unordered[tid] = shared_rows[tid] = 0;
    bad = 0;
    carry = 0;
  }
  for (int i = tid; i < 2 * kBuckets; i += kPlanThreads) hist[i / kBuckets][i % kBuckets] = 0;
  __syncthreads();
  auto blocks_of = [&](int b) {                       // single tokens: blocks of kPieceKeys keys that sequence b's token sees
    const int n = k_len[b];
    if (!inside(k_start[b], n, Tk)) return 0;
    const int seen = window > 0 ? min(n, window) : n;
    return (seen + kPieceKeys - 1) / kPieceKeys;
  };
  for (int b = tid; b < n_seq; b += kPlanThreads) {
    const int kl = k_len[b], ql = single ? 1 : q_len[b];
    if (!inside(k_start[b], kl, Tk) || (!single && !inside(q_start[b], ql, Tq)) || (prefix && prefix[b] < 0)) {
      bad = 1;
      continue;
    }
    atomicAdd(&sums[0], static_cast<unsigned long long>(single ? blocks_of(b) : ql));
    atomicAdd(&sums[1], static_cast<unsigned long long>(kl));
    if (!single && b > 0) {
      if (q_start[b] - static_cast<int64_t>(q_start[b - 1]) < q_len[b - 1]) unordered[0] = 1;
      if (k_start[b] - static_cast<int64_t>(k_start[b - 1]) < k_len[b - 1]) unordered[1] = 1;
    }
  }
  __syncthreads();
  // Rows of several sequences: query rows, or key rows in the backward, would be written by several workgroups (and need more items than there
  // is room for, where the lengths add up to more than the rows).  Sequences that each begin at or behind the end of the one before share
  // none; of others every row is marked, a bit each, in the place of the items, which has 16 words for every 64 rows or 128 (24 sequences of
  // 8192 rows: 15 us in order, 30 in another).
  if (!single && !bad)
    for (int kind = 0; kind < 2; ++kind) {
      const int rows = kind ? Tk : Tq;
      const int *start = kind ? k_start : q_start, *len = kind ? k_len : q_len;
      if (sums[kind] > static_cast<unsigned long long>(rows)) {
        if (tid == 0) shared_rows[kind] = 1;
        continue;
      }
      if (!unordered[kind]) continue;
      unsigned* marks = reinterpret_cast<unsigned*>(plan + (kind ? z.k_at : z.q_at));
      for (int i = tid; i < (rows + 31) / 32; i += kPlanThreads) marks[i] = 0;
      __threadfence();
      __syncthreads();
      for (int b = wave; b < n_seq; b += kPlanThreads / 64) {
        const int first = start[b], n = len[b];
        if (n == 0) continue;
        const int w0 = first >> 5, w1 = (first + n - 1) >> 5;
        for (int w = w0 + lane; w <= w1; w += 64) {
          unsigned mask = ~0u;
          if (w == w0) mask &= ~0u << (first & 31);
          if (w == w1) mask &= ~0u >> (31 - ((first + n - 1) & 31));
          if (atomicOr(marks + w, mask) & mask) shared_rows[kind] = 1;
        }
      }
      __threadfence();
    }
  __syncthreads();
  const bool refuse = bad || shared_rows[0];
  const bool keys_once = !refuse && !single && !shared_rows[1];                        // else no backward
  if (tid < kPlanTagWords) plan[tid] = tag.w[tid];
  if (tid == 0) {
    plan[kPlanBad] = refuse;
    plan[kPlanNoBackward] = !keys_once;
  }
  if (refuse) return;

  if (single) {
    // pieces of whole blocks, as equal as the total over the sequences allows; every sequence has one at least
    // (no sequence has more than 2^23 blocks, whatever many that share a cache add up to)
    const int per = z.target == 0 ? 1 << 23 : static_cast<int>(min(max(1ull, (sums[0] + z.target - 1) / z.target), 1ull << 23));
    for (int b0 = 0; b0 < n_seq; b0 += kPlanThreads) {
      const int b = b0 + tid;
      const int blocks = b < n_seq ? blocks_of(b) : 0, n = b < n_seq ? max(1, (blocks + per - 1) / per) : 0;
      scan[tid] = n;
      __syncthreads();
      for (int d = 1; d < kPlanThreads; d *= 2) {
        const int v = tid >= d ? scan[tid - d] : 0;
        __syncthreads();
        scan[tid] += v;
        __syncthreads();
      }
      const int first = carry + scan[tid] - n;
      if (b < n_seq) {
        const int kl = k_len[b], lo = window > 0 ? max(0, kl - window) : 0;
        plan[z.seq_at + 2 * b] = first;
        plan[z.seq_at + 2 * b + 1] = n;
        for (int i = 0; i < n; ++i) {
          const int j0 = lo + i * per * kPieceKeys, j1 = i + 1 < n ? j0 + per * kPieceKeys : kl;
          int* w = plan + z.q_at + kItemWords * (first + i);
          w[0] = b;
          w[1] = k_start[b] + j0;
          w[2] = j1 - j0;
          w[3] = kl - 1 - j0;                          // distance of the piece's first key
          w[4] = n;
        }
      }
      __syncthreads();
      if (tid == kPlanThreads - 1) carry = first + n;
      __syncthreads();
    }
    if (tid == 0) {
      plan[kPlanQItems] = carry;
      plan[kPlanKItems] = 0;
    }
    return;
  }

  // Passes over all tiles, a wavefront a sequence and a lane a tile: what they cost in all; the items of each cost, counted; the items,
  // placed, the most expensive first.  A tile that costs more than a slot's share of the device is cut into pieces of equal length along
  // what its workgroup walks (keys; query heads and queries), which leave float32 sums for the join kernels.  A piece is 8 blocks of 64
  // at least, and there are at most z.extra_* more pieces than tiles.  Items of one cost, and the places of sums, come in no particular
  // order; no result depends on it.
  const int rep = tag.w[kTagNq] / tag.w[kTagNkv];
  // a wavefront a sequence; of few sequences, all wavefronts share the tiles of each
  const int stride = n_seq < kPlanThreads / 64 ? kPlanThreads : 64, lead = stride == 64 ? lane : tid;
  for (int pass = -1; pass < 2; ++pass) {
    unsigned long long sum[2] = {0, 0};
    int longest_seen[2] = {0, 0};
    for (int b = stride == 64 ? wave : 0; b < n_seq; b += stride == 64 ? kPlanThreads / 64 : 1) {
      const int ql = q_len[b], kl = k_len[b], qs = q_start[b], ks = k_start[b], off = kl - ql;
      const int pre = prefix ? min(prefix[b], kl) : 0;
      auto tile = [&](int kind, int row0, int rows, int from, int to, auto&& fill) {
        const int len = to - from;
        if (pass < 0) {
          sum[kind] += len;
          longest_seen[kind] = max(longest_seen[kind], len);
          return;
        }
        const int pieces = len <= most_of_piece[kind] ? 1 : (len + most_of_piece[kind] - 1) / most_of_piece[kind];
        const int each = pieces == 1 ? len : len / pieces, more = pieces == 1 ? 0 : len - each * pieces;      // the first `more` are one longer
        int slot = -1;
        if (pass == 1 && pieces > 1) {
          slot = atomicAdd(&slots[kind], pieces);
          int* w = plan + z.join_at[kind] + 8 * atomicAdd(&joins[kind], 1);
          w[0] = row0; w[1] = rows; w[2] = slot; w[3] = pieces;
        }
        for (int i = 0; i < pieces; ++i) {
          const int p0 = from + i * each + min(i, more), p1 = p0 + each + (i < more ? 1 : 0);
          // 0: the most expensive; the product is below kBuckets for every cost up to the longest, whatever its rounding
          const int bucket = kBuckets - 1 - min(kBuckets - 1, static_cast<int>(static_cast<float>(p1 - p0) * per_cost[kind]));
          const int at = atomicAdd(&hist[kind][bucket], 1);
          if (pass == 1) fill(plan + (kind ? z.k_at : z.q_at) + kItemWords * at, p0, p1, slot < 0 ? -1 : slot + i);
        }
      };
      for (int t = lead; t < (ql + 127) / 128; t += stride) {
        const int r0 = 128 * t, n = min(128, ql - r0), p = off + r0;
        const int lo = keys_of(p, kl, pre, window, causal).lo, hi = keys_of(p + n - 1, kl, pre, window, causal).hi;
        tile(0, qs + r0, n, hi > lo ? lo / kTok : 0, hi > lo ? (hi + kTok - 1) / kTok : 0, [&](int* w, int b0, int b1, int slot) {
          w[0] = qs + r0; w[1] = n; w[2] = p; w[3] = ks; w[4] = kl; w[5] = pre; w[6] = b0; w[7] = b1; w[8] = slot;
        });
      }
      if (!keys_once) continue;
      for (int t = lead; t < (kl + kTok - 1) / kTok; t += stride) {
        const int k0 = kTok * t, n = min(kTok, kl - k0);
        const int lo = queries_of(k0, ql, off, pre, window, causal).lo, hi = queries_of(k0 + n - 1, ql, off, pre, window, causal).hi;
        const int blocks = hi > lo ? (hi + kTok - 1) / kTok - lo / kTok : 0;
        tile(1, ks + k0, n, 0, rep * blocks, [&](int* w, int s0, int s1, int slot) {
          w[0] = ks + k0; w[1] = n; w[2] = k0; w[3] = qs; w[4] = ql; w[5] = off; w[6] = pre; w[7] = s0; w[8] = s1; w[9] = slot;
        });
      }
    }
    if (pass < 0)
      for (int kind = 0; kind < 2; ++kind)
        if (sum[kind]) {
          atomicAdd(&total[kind], sum[kind]);
          atomicMax(&longest[kind], longest_seen[kind]);
        }
    __syncthreads();
    if (tid < 2) {
      const int extra = tid == 0 ? z.extra_q : z.extra_k;
      if (pass < 0) {
        const unsigned long long share = extra > 0 ? (total[tid] + extra - 1) / extra : 0x7FFFFFFFull;
        most_of_piece[tid] = static_cast<int>(min(max(share, static_cast<unsigned long long>(kLeastPiece)), 1ull << 30));
        per_cost[tid] = static_cast<float>(kBuckets) / static_cast<float>(min(longest[tid], most_of_piece[tid]) + 1);
      } else if (pass == 0) {                          // counts -> first place of each cost
        int at = 0;
        for (int i = 0; i < kBuckets; ++i) {
          const int n = hist[tid][i];
          hist[tid][i] = at;
          at += n;
        }
        plan[tid == 0 ? kPlanQItems : kPlanKItems] = at;
      } else {
        plan[tid == 0 ? kPlanQJoins : kPlanKJoins] = joins[tid];
      }
    }
    __syncthreads();
  }
}

// x, in a way that the compiler cannot carry over from an earlier place: what is cheap to form again does not occupy registers in between
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A workgroup's look at the plan: one load brings the header (lanes 0 .. 15) and the words of its item (16 .. 31), which lie inside the
// plan's memory whether or not that many items are in use
template <int WORDS>
struct PlanLook {
  int w;
  __device__ __forceinline__ PlanLook(const int* __restrict__ plan, int items_at, int item, int lane)
      : w(plan[lane < 16 ? lane : items_at + WORDS * item + (lane & (WORDS - 1))]) {}
  __device__ __forceinline__ int header(int i) const { return __builtin_amdgcn_readlane(w, i); }
  __device__ __forceinline__ int item(int i) const { return __builtin_amdgcn_readlane(w, 16 + i); }
  // Is this the plan of the call's description?  What is not is answered with NaN.
  __device__ __forceinline__ bool is(const PlanTag& tag, bool backward) const {
    bool ok = header(kPlanBad) == 0 && !(backward && header(kPlanNoBackward) != 0);
#pragma unroll
    for (int i = 0; i < kPlanTagWords; ++i) ok = ok && header(i) == tag.w[i];
    return ok;
  }
};
typedef PlanLook<kItemWords> PlanWords;
__device__ __forceinline__ void fill_nan(bf16_t* p, int64_t rows, int64_t width, int64_t ld) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < width; c += blockDim.x) p[r * ld + c] = 0x7FC0;
}
__device__ __forceinline__ void fill_nan(float* p, int64_t n) {
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = __uint_as_float(0x7FC00000u);
}

// ---- scores ---------------------------------------------------------------------------------------------------------------------
struct Scores {
  float c;             // scale log2(e): z in units of log 2
  float a, b;          // capped: a = cap log2(e); tanh(z / cap) = 1 - 2 / (1 + 2^(b q.k))
  float t;             // scale / cap
  float ref;           // kBounded: the fixed reference of the exponents
  float slope;         // slope log2(e)
};
__device__ __forceinline__ Scores scores_of(const MaskedDims& d, int head, bool biased) {
  return {d.c, d.cap_a, d.cap_b, d.cap_t, d.ref, biased && d.slopes ? d.slopes[head] * kLog2e : 0.0f};
}
// from a reference maximum (units of log 2) and the sum of 2^(score - it): -inf where there is no key; a NaN stays one
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -INFINITY : m * kLn2 + logf(l); }
// 1 / (1 + 2^(b q.k)) = (1 - tanh) / 2
__device__ __forceinline__ float cap_half(const Scores& sc, float x) {
  return __builtin_amdgcn_rcpf(1.0f + fast_exp2(x * sc.b));
}
// Wide caps.  a - 2 a cap_half is a difference of two numbers near a wherever |z| is far below the cap, and off by up to 2^-22 a whatever the
// score: 2e-5 at a cap of 50, and at one of 1e8 a score of 20 drowns in it.  Up to a = kNarrow (a cap of 709) that is below 2^-12, a
// sixteenth of the half step to which a probability is rounded next.  Beyond, while |z / cap| < 1/4, the score is z tanh(t) / t, t = z / cap, by
// the series in t^2 up to t^8 (the next term is 8e-9 at 1/4), and else a (1 - 2 cap_half), which there is good to 16 half-steps of itself.  8192
// causal tokens, 16 / 8 heads of 128, forward and backward in us: a cap of 100 this way 500 and 1468, the narrow way 371 and 1103; of 1000
// this way 399 and 1389 (heads of 64: 271 and 891, the narrow way 285 and 674).
constexpr float kNarrow = 1024.0f;
__device__ __forceinline__ float tanh_over(float u) {
  const float w = (u - 2.4677419f) * (62.0f / 2835.0f);                        // 62/2835 u - 17/315
  return fmaf(u, fmaf(u, fmaf(u, w, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
}
// is any of the wavefront's scores beyond?  (a NaN is)
template <int N>
__device__ __forceinline__ bool any_far(const Scores& sc, const f32x16 (&x)[N]) {
  float top = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(x[k][v]));
  return __any(!(top * sc.t < 0.25f));
}
// kFar: some may be beyond.  r: (1 - tanh) / 2
template <bool kFar>
__device__ __forceinline__ float wide_score(const Scores& sc, float x, float& r) {
  const float t = x * sc.t, u = t * t, g = tanh_over(u);
  float y = x * sc.c * g;
  r = fmaf(-0.5f * t, g, 0.5f);
  if constexpr (kFar) {
    const float far = cap_half(sc, x);
    r = u < 0.0625f ? r : far;
    y = u < 0.0625f ? y : sc.a * fmaf(-2.0f, far, 1.0f);
  }
  return y;
}

// ---- forward --------------------------------------------------------------------------------------------------------------------
template <class H>
struct MaskedState {
  bf16x8 qf[H::KS];
  f32x16 oacc[H::DT];   // rows = dh, column = query lane % 32
  float mc, l, lr;        // reference maximum (units of log 2), this half-wave's share of the denominator, and that of rounded probabilities
};

// a + the two bf16 of w
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float add_pair(uint32_t w, float a) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), a, false);
}

// NT x 32 keys of tiles at k_lds, v_lds (first 32: half `h0`).  first: index of the lane's first key relative to what is compared:
// `len` keys from 0 on are seen (masked); last: heads are so wide that the last step of 16 columns of q.k counts (uses_last); gap: distance of the lane's first key from its query.
template <class H, int kMode, int NT>
__device__ __forceinline__ void masked_block(MaskedState<H>& st, uint32_t k_lds, uint32_t v_lds, uint32_t ra, uint32_t ca, const Scores& sc,
                                             int h0, bool last, bool masked, int first, int len, float gap, bool raw) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  typedef Tile<DH> Tl;
  f32x16 s[NT];            // rows = keys, column = query
#pragma unroll
  for (int kt = 0; kt < NT; ++kt) s[kt] = zero16();
  // Operands from LDS are requested kRing - 1 matrix instructions ahead, and the first of V's before the exponents, during which they
  // arrive; scheduling barriers keep the order.
  constexpr int kRing = 6, kFirst = 4, kQK = NT * KS, kPV = NT * 2 * DT;
  bf16x8 f[kRing];
  auto fetch_k = [&](int i) { f[i % kRing] = Tl::rows(k_lds + ra, h0 + i % NT, i / NT); };
#pragma unroll
  for (int i = 0; i < kRing - 1 && i < kQK; ++i) fetch_k(i);
#pragma unroll
  for (int i = 0; i < kQK - NT; ++i) {
    if (i + kRing - 1 < kQK) fetch_k(i + kRing - 1);
    s[i % NT] = mfma(f[i % kRing], st.qf[i / NT], s[i % NT]);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (last) {
#pragma unroll
    for (int i = kQK - NT; i < kQK; ++i) s[i % NT] = mfma(f[i % kRing], st.qf[i / NT], s[i % NT]);
  }
  auto fetch_v = [&](int i) { f[i % kRing] = Tl::cols(v_lds + ca, h0 + i / (2 * DT), i / DT % 2, i % DT); };
#pragma unroll
  for (int i = 0; i < kFirst; ++i) fetch_v(i);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (kMode == kWide) {
    float r;
    if (any_far(sc, s)) {
#pragma unroll
      for (int i = 0; i < NT * 16; ++i) {
        float x = s[i / 16][i % 16];
        asm("" : "+v"(x));             // else what the two branches share is formed for all scores before them: registers
        s[i / 16][i % 16] = wide_score<true>(sc, x, r);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NT * 16; ++i) s[i / 16][i % 16] = wide_score<false>(sc, s[i / 16][i % 16], r);
    }
  }
#pragma unroll
  for (int kt = 0; kt < NT; ++kt)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int j = 32 * kt + 8 * (v / 4) + v % 4;     // + 4 (lane / 32), which first and gap hold
      float x = s[kt][v];
      if constexpr (kMode == kBounded) x = fmaf(-2.0f * sc.a, cap_half(sc, x), sc.a - sc.ref);
      if constexpr (kMode == kCapped) x = fmaf(-2.0f * sc.a, cap_half(sc, x), sc.a);
      if constexpr (kMode == kBiased) x = x * sc.c;
      if constexpr (kMode == kBiased || kMode == kCapped || kMode == kWide) x = fmaf(-sc.slope, fabsf(gap - static_cast<float>(j)), x);
      s[kt][v] = x;
    }
  if (masked) {
#pragma unroll
    for (int kt = 0; kt < NT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        s[kt][v] = static_cast<uint32_t>(first + 32 * kt + 8 * (v / 4) + v % 4) < static_cast<uint32_t>(len) ? s[kt][v] : -INFINITY;
  }
  if constexpr (DH == 128 && (kMode == kBiased || kMode == kCapped || kMode == kWide)) __builtin_amdgcn_sched_barrier(0);   // registers
  if constexpr (kMode != kBounded) {
    float mx = s[0][0];
#pragma unroll
    for (int kt = 0; kt < NT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kt][v]);
    mx = half_max(mx);
    if constexpr (kMode == kPlain) mx *= sc.c;
    if (__any(mx > st.mc + kLazy)) {
      const float nm = fmaxf(st.mc, mx);
      const float alpha = fast_exp2(st.mc - nm);
      st.mc = nm;
      st.l *= alpha;
      st.lr *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) st.oacc[dt] *= alpha;
    }
  }
  float ps = 0.0f;
#pragma unroll
  for (int kt = 0; kt < NT; ++kt)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      float p;
      if constexpr (kMode == kPlain) p = fast_exp2(fmaf(s[kt][v], sc.c, -st.mc));
      else if constexpr (kMode == kBounded) p = fast_exp2(s[kt][v]);
      else p = fast_exp2(s[kt][v] - st.mc);
      s[kt][v] = p;
    }
  if (raw) {
#pragma unroll
    for (int kt = 0; kt < NT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) ps += s[kt][v];
    st.l += ps;
  }
  Frag p[NT][2];
#pragma unroll
  for (int kt = 0; kt < NT; ++kt) {
    p[kt][0].v = pack8<0>(s[kt]);
    p[kt][1].v = pack8<1>(s[kt]);
#pragma unroll
    for (int i = 0; i < 4; ++i) st.lr = add_pair(p[kt][1].w[i], add_pair(p[kt][0].w[i], st.lr));
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = kFirst; i < kRing - 1 && i < kPV; ++i) fetch_v(i);
#pragma unroll
  for (int i = 0; i < kPV; ++i) {
    if (i + kRing - 1 < kPV) fetch_v(i + kRing - 1);
    st.oacc[i % DT] = mfma(f[i % kRing], p[i / (2 * DT)][i / DT % 2].v, st.oacc[i % DT]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// what rounding four floats to bf16 (w) took from them, in units of 2^-8 of the last place: a signed byte each
__device__ __forceinline__ uint32_t low_bytes(const float (&x)[4], const uint2& w) {
  const uint32_t top[4] = {w.x << 16, w.x & 0xFFFF0000u, w.y << 16, w.y & 0xFFFF0000u};
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int off = static_cast<int>(__float_as_uint(x[i]) - top[i]);            // -2^15 .. 2^15
    r |= static_cast<uint32_t>(min(127, (off + 128) >> 8) & 0xFF) << (8 * i);
  }
  return r;
}
// A wavefront's 32 rows x DH results, which lie across its lanes (lane n, half hi: row n, columns 32 dt + 8 j + 4 hi + 0..3), go through LDS
// and leave as 16 bytes a lane, a row after the other: stored as they lie, 8 bytes of 32 rows an instruction, they take 23 us instead
// of 8 (8192 rows of 16 heads of 128, with the low bytes).  Rows are padded by 16 bytes.
template <int DH>
struct RowStage {
  static constexpr int PITCH = DH * 2 + 16, LOW_PITCH = DH + 16, BYTES = 32 * (PITCH + LOW_PITCH);
  static __device__ __forceinline__ void put(char* at, int lane, int dt, int j, const float (&x)[4], bool low) {
    const int n = lane & 31, col = 32 * dt + 8 * j + 4 * (lane >> 5);
    const uint2 w = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    *reinterpret_cast<uint2*>(at + n * PITCH + col * 2) = w;
    if (low) *reinterpret_cast<uint32_t*>(at + 32 * PITCH + n * LOW_PITCH + col) = low_bytes(x, w);
  }
  // rows rows (of 32) and dh columns to out, `ld` elements apart, and the low bytes to out_low, ld_low apart
  static __device__ __forceinline__ void flush(const char* at, int lane, int rows, int dh, bf16_t* out, int64_t ld, uint8_t* out_low, int64_t ld_low) {
    constexpr int CPR = DH / 8, RPP = 64 / CPR;        // chunks per row, rows per pass
    const int chunk = lane % CPR;
#pragma unroll
    for (int i = 0; i < 32 / RPP; ++i) {
      const int row = i * RPP + lane / CPR;
      if (row >= rows || chunk * 8 >= dh) continue;
      *reinterpret_cast<uint4*>(out + row * ld + chunk * 8) = *reinterpret_cast<const uint4*>(at + row * PITCH + chunk * 16);
      if (out_low)
        *reinterpret_cast<uint2*>(out_low + row * ld_low + chunk * 8) =
            *reinterpret_cast<const uint2*>(at + 32 * PITCH + row * LOW_PITCH + chunk * 8);
    }
  }
};

// a wavefront's 32 rows x dh as float32 sums of a piece, rows dh apart
template <class H>
__device__ __forceinline__ void leave_sums(const f32x16 (&acc)[H::DT], float* out, int rows, int dh, int lane) {
  const int n = lane & 31, hi = lane >> 5;
  if (n >= rows) return;
#pragma unroll
  for (int dt = 0; dt < H::DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (dt * 32 + 8 * j < dh)
        *reinterpret_cast<float4*>(out + n * dh + dt * 32 + 8 * j + 4 * hi) = make_float4(acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]);
}

// the float of a bf16 and its byte
__device__ __forceinline__ float with_low(uint32_t bf16_top, uint32_t byte) {
  return __uint_as_float(bf16_top + (static_cast<uint32_t>(static_cast<int>(byte << 24) >> 24) << 8));
}

// A workgroup: 128 queries of one head, 32 a wavefront (the columns of S^T = K Q^T, so that a lane holds scores of one query), and the blocks
// of 64 keys that any of them sees.  Matrix cores and vector unit share a SIMD's issue (a product of 32 cycles takes 16 of it), and
// the chip its power: 16384 tokens behind a prefix, 16 / 8 heads of 128, capped: 1205-1240 us (1250 and more before the clock has settled), 0.9-0.93 PFLOP/s of
// what the masks leave (products and LDS alone 836).  24 documents in 8192 tokens: 50 us, by the first loads of short items.
template <class H, int kMode>
__global__ void __launch_bounds__(256, 2)
k_masked_fwd(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const int* __restrict__ plan, PlanTag tag,
             PlanSizes z, MaskedDims d, bf16_t* __restrict__ O, float* __restrict__ lse, uint8_t* __restrict__ o_low, float* __restrict__ part) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  typedef Tile<DH> Tl;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][Tl::ELEMS];   // [stage][k, v]
  const int item = blockIdx.x / d.n_q, pair = blockIdx.x % d.n_q;
  const PlanWords w(plan, z.q_at, item, threadIdx.x & 63);
  if (!w.is(tag, false)) {
    fill_nan(O, d.Tq, (int64_t)d.n_q * d.dh, d.ldo);
    if (lse) fill_nan(lse, d.Tq * d.n_q);
    return;
  }
  if (item >= w.header(kPlanQItems)) return;
  const int row0 = w.item(0), rows = w.item(1), pos0 = w.item(2), k_start = w.item(3), k_len = w.item(4), prefix = w.item(5);
  const int kb0 = w.item(6), kb1 = w.item(7), slot = w.item(8);
  const int window = tag.w[kTagWindow];
  const bool causal = tag.w[kTagFlags] & 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hi = lane >> 5;
  const int kvh = pair % d.n_kv, head = kvh * (d.n_q / d.n_kv) + pair / d.n_kv;
  const Scores sc = scores_of(d, head, kMode == kBiased || kMode == kCapped || kMode == kWide);

  const int mine = min(32, rows - 32 * wave);          // this wavefront's queries (none: <= 0)
  const bool live = n < mine;
  const int p = pos0 + 32 * wave + n;
  const Seen seen = live ? keys_of(p, k_len, prefix, window, causal) : Seen{0, 0};
  const Seen sa = keys_of(pos0 + 32 * wave, k_len, prefix, window, causal), sb = keys_of(pos0 + 32 * wave + mine - 1, k_len, prefix, window, causal);

  MaskedState<H> st;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    st.qf[ks] = live && ks * 16 + 8 * hi < d.dh ? load_frag16(Q + ((int64_t)row0 + 32 * wave + n) * d.ldq + head * d.dh + ks * 16 + 8 * hi) : bf16x8{};
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) st.oacc[dt] = zero16();
  st.mc = kMode == kBounded ? sc.ref : kLowest;
  st.l = st.lr = 0.0f;
  const int64_t kvcol = (int64_t)kvh * d.dh;
  const uint32_t lds0 = lds_addr_of(lds), ra = Tl::rows_at(lane), ca = Tl::cols_at(lane);
  const bool last = uses_last<H>(d.dh);
  const uint32_t from_k = Tl::of_lane(d.ldk, tid), from_v = Tl::of_lane(d.ldv, tid);
  auto request = [&](int kb) {
    const uint32_t at = lds0 + (kb & 1) * (2 * Tl::ELEMS * 2);
    copy_tile<DH>(K, (int64_t)k_start + kb * kTok, k_len - kb * kTok, d.ldk, kvcol, d.dh, from_k, at, wave, tid);
    copy_tile<DH>(V, (int64_t)k_start + kb * kTok, k_len - kb * kTok, d.ldv, kvcol, d.dh, from_v, at + Tl::ELEMS * 2, wave, tid);
  };
  clear_columns<H>(&lds[0][0][0], 4, d.dh, tid);
  if (kb0 < kb1) request(kb0);
  for (int kb = kb0; kb < kb1; ++kb) {
    FAAR_WAIT_VMCNT(0);                                // block kb has landed (mine); the barrier: everybody's, and nobody reads
    __syncthreads();                                   // the other stage any more
    if (kb + 1 < kb1) request(kb + 1);
    const uint32_t k_lds = lds0 + (kb & 1) * (2 * Tl::ELEMS * 2), v_lds = k_lds + Tl::ELEMS * 2;
    const int k0 = kb * kTok;
    if (mine <= 0 || k0 >= sb.hi || k0 + kTok <= sa.lo) continue;
    const float gap = static_cast<float>(p - k0 - 4 * hi);
    masked_block<H, kMode, 2>(st, k_lds, v_lds, ra, ca, sc, 0, last, !(k0 >= sb.lo && k0 + kTok <= sa.hi), k0 + 4 * hi - seen.lo,
                               max(0, seen.hi - seen.lo), gap, lse != nullptr);
  }
  __syncthreads();                                     // the tiles have been read: their place is free
  if (mine <= 0) return;
  const float lt = half_sum(st.l), lr = half_sum(st.lr);
  if (slot >= 0) {                                     // a piece: [128 rows][dh] sums, then maximum and denominators of the rows
    float* at = part + ((int64_t)slot * d.n_q + head) * (128 * (d.dh + kPartExtra));
    leave_sums<H>(st.oacc, at + 32 * wave * d.dh, mine, d.dh, lane);
    float* m = at + 128 * d.dh + 32 * wave + n;
    if (hi == 0 && n < mine) {
      m[0] = st.mc;
      m[128] = lt;
      m[256] = lr;
    }
    return;
  }
  const float inv = lr == 0.0f ? 0.0f : 1.0f / lr;     // a query that sees no key: 0; a NaN stays one
  char* stage = reinterpret_cast<char*>(lds) + wave * RowStage<DH>::BYTES;
  static_assert(4 * RowStage<DH>::BYTES <= sizeof(lds), "rows fit in the stages");
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = st.oacc[dt][4 * j + r] * inv;
      RowStage<DH>::put(stage, lane, dt, j, x, o_low != nullptr);
    }
  const int64_t t = (int64_t)row0 + 32 * wave, width = (int64_t)d.n_q * d.dh;
  if (lse && hi == 0 && n < mine) lse[(int64_t)head * d.Tq + t + n] = lse_of(st.mc, lt);
  RowStage<DH>::flush(stage, lane, mine, d.dh, O + t * d.ldo + head * d.dh, d.ldo, o_low ? o_low + t * width + head * d.dh : nullptr, width);
}

// the pieces of a tile's queries, in their order; one query head a workgroup
__global__ void __launch_bounds__(kJoinThreads)
k_masked_join_fwd(const int* __restrict__ plan, PlanTag tag, PlanSizes z, MaskedDims d, const float* __restrict__ part, bf16_t* __restrict__ O,
                  float* __restrict__ lse, uint8_t* __restrict__ o_low) {
  const int item = blockIdx.x / d.n_q, head = blockIdx.x % d.n_q;
  const PlanLook<8> w(plan, z.join_at[0], item, threadIdx.x & 63);
  if (!w.is(tag, false) || item >= w.header(kPlanQJoins)) return;      // a wrong plan: answered by the kernel before
  const int64_t row0 = w.item(0), step = (int64_t)d.n_q * 128 * (d.dh + kPartExtra), width = (int64_t)d.n_q * d.dh;
  const int rows = w.item(1), pieces = w.item(3), c4 = d.dh / 4;
  const float* first = part + ((int64_t)w.item(2) * d.n_q + head) * (128 * (d.dh + kPartExtra));
  for (int i = threadIdx.x; i < rows * c4; i += kJoinThreads) {
    const int row = i / c4, col = i % c4 * 4;
    const float *sums = first + row * d.dh + col, *stats = first + 128 * d.dh + row;
    float m = kLowest, l = 0.0f, r = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < pieces; ++p) m = fmaxf(m, stats[p * step]);
#pragma unroll 2
    for (int p = 0; p < pieces; ++p) {
      const float f = fast_exp2(stats[p * step] - m);
      const float4 v = *reinterpret_cast<const float4*>(sums + p * step);
      l += stats[p * step + 128] * f;
      r += stats[p * step + 256] * f;
      x[0] += v.x * f; x[1] += v.y * f; x[2] += v.z * f; x[3] += v.w * f;
    }
    const float inv = r == 0.0f ? 0.0f : 1.0f / r;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= inv;
    const uint2 o = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    *reinterpret_cast<uint2*>(O + (row0 + row) * d.ldo + head * d.dh + col) = o;
    if (o_low) *reinterpret_cast<uint32_t*>(o_low + (row0 + row) * width + head * d.dh + col) = low_bytes(x, o);
    if (lse && col == 0) lse[(int64_t)head * d.Tq + row0 + row] = lse_of(m, l);
  }
}

// ---- backward: dq ---------------------------------------------------------------------------------------------------------------
// x: q.k of an element -> its probability, with `shift` what a query's scores are shifted by (in units of log 2; under a narrow cap: the cap
// less lse, else -lse); and a quarter of what the cap leaves of a gradient: with r = (1 - tanh) / 2, 1 - tanh^2 = 4 (r - r^2).  The 4 is
// in d.grad_scale.
template <int kCap, bool kBias>
__device__ __forceinline__ float prob_of(float x, const Scores& sc, float shift, float gap, float& slack) {
  float y;
  if constexpr (kCap == kNarrowCap) {
    const float r = cap_half(sc, x);
    slack = fmaf(-r, r, r);
    y = fmaf(-2.0f * sc.a, r, shift);
  } else if constexpr (kCap == kWideCap) {             // x is the score already
    y = x + shift;
  } else {
    y = fmaf(x, sc.c, shift);
  }
  if constexpr (kBias) y = fmaf(-sc.slope, fabsf(gap), y);
  return fast_exp2(y);
}

// Wide caps: q.k of a tile become scores, and what the cap leaves of their gradients is multiplied into dP - delta: one after the other, in
// place.  kLook: a tile that has no score beyond leaves the exponentials out (dk and dv of heads of 128 lack the registers to look)
template <bool kLook>
__device__ __forceinline__ void wide_scores(const Scores& sc, f32x16& s, f32x16& dp) {
  const bool far = !kLook || any_far(sc, reinterpret_cast<const f32x16(&)[1]>(s));
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    float r, x = s[v];
    if (far) {
      if constexpr (kLook) asm volatile("" : "+v"(x));   // keeps what the branches share from being formed for all scores before them
      x = wide_score<true>(sc, x, r);
    } else {
      x = wide_score<false>(sc, x, r);
    }
    s[v] = x;
    dp[v] *= fmaf(-r, r, r);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// 32 keys (half kt of the tiles).  The operands from LDS pass through a ring of kRing, each requested kRing - 1 matrix instructions
// ahead, as in the dk / dv kernel, and for its reason: with all of them requested at once registers run out.
template <class H, int kCap, bool kBias>
__device__ __forceinline__ void masked_dq_tile(f32x16 (&acc)[H::DT], const bf16x8 (&qf)[H::KS], const bf16x8 (&dof)[H::KS], float shift,
                                               const f32x16& less, uint32_t k_rows, uint32_t v_rows, uint32_t k_cols, const Scores& sc, bool last, bool masked,
                                               int first, int len, float gap) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  typedef Tile<DH> Tl;
  constexpr int kRing = 4;
  bf16x8 f[kRing];
  f32x16 s = zero16(), dp = less;          // rows = keys, column = query; dP starts at -delta, which saves the subtraction
  auto fetch_rows = [&](int i) { f[i % kRing] = Tl::rows(i & 1 ? v_rows : k_rows, 0, i / 2); };
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) fetch_rows(i);
#pragma unroll
  for (int i = 0; i < 2 * KS - 2; ++i) {
    if (i + kRing - 1 < 2 * KS) fetch_rows(i + kRing - 1);
    if (i % 2 == 0) s = mfma(f[i % kRing], qf[i / 2], s);
    else dp = mfma(f[i % kRing], dof[i / 2], dp);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (last) {
    s = mfma(f[(2 * KS - 2) % kRing], qf[KS - 1], s);
    dp = mfma(f[(2 * KS - 1) % kRing], dof[KS - 1], dp);
  }
  if constexpr (kCap == kWideCap) wide_scores<true>(sc, s, dp);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int j = 8 * (v / 4) + v % 4;
    float slack = 1.0f;
    float p = prob_of<kCap, kBias>(s[v], sc, shift, gap - static_cast<float>(j), slack);
    dp[v] *= p;
    if constexpr (kCap == kNarrowCap) dp[v] *= slack;
  }
  if (masked) {
#pragma unroll
    for (int v = 0; v < 16; ++v) dp[v] = static_cast<uint32_t>(first + 8 * (v / 4) + v % 4) < static_cast<uint32_t>(len) ? dp[v] : 0.0f;
  }
  const bf16x8 df[2] = {pack8<0>(dp), pack8<1>(dp)};
  __builtin_amdgcn_sched_barrier(0);
  auto fetch_cols = [&](int i) { f[i % kRing] = Tl::cols(k_cols, 0, i / DT, i % DT); };
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) fetch_cols(i);
#pragma unroll
  for (int i = 0; i < 2 * DT; ++i) {
    if (i + kRing - 1 < 2 * DT) fetch_cols(i + kRing - 1);
    acc[i % DT] = mfma(f[i % kRing], df[i / DT], acc[i % DT]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The forward's split, walked again: S and dP = V dO^T in tiles of 32 keys, dq^T += K^T dz^T.  Bound like the forward, by a query's four operands
// on short sequences: 8192 causal tokens, 16 / 8 heads of 128, 374 us (scores of deviation 1) to 423 (9), 479 capped; 24 documents
// of 8192 tokens 71, of which vector unit 27 and matrix cores 13.
template <class H, int kCap, bool kBias>
__global__ void __launch_bounds__(256, 2)
k_masked_bwd_dq(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const bf16_t* __restrict__ dO,
                const bf16_t* __restrict__ O, const uint8_t* __restrict__ o_low, const float* __restrict__ lse, const int* __restrict__ plan, PlanTag tag,
                PlanSizes z, MaskedDims d, float* __restrict__ delta, bf16_t* __restrict__ dQ, float* __restrict__ part) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  typedef Tile<DH> Tl;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][Tl::ELEMS];   // [stage][k, v]
  const int item = blockIdx.x / d.n_q, pair = blockIdx.x % d.n_q;
  const PlanWords w(plan, z.q_at, item, threadIdx.x & 63);
  if (!w.is(tag, true)) {
    fill_nan(dQ, d.Tq, (int64_t)d.n_q * d.dh, d.ldq);
    return;
  }
  if (item >= w.header(kPlanQItems)) return;
  const int row0 = w.item(0), rows = w.item(1), pos0 = w.item(2), k_start = w.item(3), k_len = w.item(4), prefix = w.item(5);
  const int kb0 = w.item(6), kb1 = w.item(7), slot = w.item(8);
  const int window = tag.w[kTagWindow];
  const bool causal = tag.w[kTagFlags] & 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hi = lane >> 5;
  const int kvh = pair % d.n_kv, head = kvh * (d.n_q / d.n_kv) + pair / d.n_kv;
  const Scores sc = scores_of(d, head, kBias);

  const int mine = min(32, rows - 32 * wave);
  const bool live = n < mine;
  const int p = pos0 + 32 * wave + n;
  const Seen seen = live ? keys_of(p, k_len, prefix, window, causal) : Seen{0, 0};
  const Seen sa = keys_of(pos0 + 32 * wave, k_len, prefix, window, causal), sb = keys_of(pos0 + 32 * wave + mine - 1, k_len, prefix, window, causal);
  const int64_t t0 = (int64_t)row0 + 32 * wave + n;

  const int64_t kvcol = (int64_t)kvh * d.dh;
  const uint32_t lds0 = lds_addr_of(lds), ra = Tl::rows_at(lane), ca = Tl::cols_at(lane);
  const bool last = uses_last<H>(d.dh);
  const uint32_t from_k = Tl::of_lane(d.ldk, tid), from_v = Tl::of_lane(d.ldv, tid);
  auto request = [&](int kb) {
    const uint32_t at = lds0 + (kb & 1) * (2 * Tl::ELEMS * 2);
    copy_tile<DH>(K, (int64_t)k_start + kb * kTok, k_len - kb * kTok, d.ldk, kvcol, d.dh, from_k, at, wave, tid);
    copy_tile<DH>(V, (int64_t)k_start + kb * kTok, k_len - kb * kTok, d.ldv, kvcol, d.dh, from_v, at + Tl::ELEMS * 2, wave, tid);
  };
  clear_columns<H>(&lds[0][0][0], 4, d.dh, tid);
  if (kb0 < kb1) request(kb0);
  bf16x8 qf[KS], dof[KS];
  float shift = 0.0f, dl = 0.0f;
  const float lse0 = live ? lse[(int64_t)head * d.Tq + t0] : 0.0f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const bool on = live && ks * 16 + 8 * hi < d.dh;
    const int64_t at = head * d.dh + ks * 16 + 8 * hi;
    qf[ks] = on ? load_frag16(Q + t0 * d.ldq + at) : bf16x8{};
    dof[ks] = on ? load_frag16(dO + t0 * d.ldo + at) : bf16x8{};
    Frag of;
    of.v = on ? load_frag16(O + t0 * d.ldo + at) : bf16x8{};
    uint2 low = make_uint2(0, 0);
    if (on && o_low) low = *reinterpret_cast<const uint2*>(o_low + t0 * ((int64_t)d.n_q * d.dh) + at);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      dl += static_cast<float>(dof[ks][j]) * with_low(j & 1 ? of.w[j / 2] & 0xFFFF0000u : of.w[j / 2] << 16, (j < 4 ? low.x : low.y) >> (8 * (j & 3)));
  }
  dl = half_sum(dl);
  if (live) {
    shift = (kCap == kNarrowCap ? sc.a : 0.0f) - lse0 * kLog2e;
    if (hi == 0) {
      delta[(int64_t)head * d.Tq + t0] = -dl;
      delta[((int64_t)d.n_q + head) * d.Tq + t0] = shift;
    }
  }
  f32x16 acc[DT], less;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = zero16();
#pragma unroll
  for (int v = 0; v < 16; ++v) less[v] = -dl;
  for (int kb = kb0; kb < kb1; ++kb) {
    FAAR_WAIT_VMCNT(0);
    __syncthreads();
    if (kb + 1 < kb1) request(kb + 1);
    const uint32_t k_lds = lds0 + (kb & 1) * (2 * Tl::ELEMS * 2), v_lds = k_lds + Tl::ELEMS * 2;
    const int k0 = kb * kTok;
    if (mine <= 0 || k0 >= sb.hi || k0 + kTok <= sa.lo) continue;
    const float gap = static_cast<float>(p - k0 - 4 * hi);
    const bool whole = k0 >= sb.lo && k0 + kTok <= sa.hi;
    const int first = k0 + 4 * hi - seen.lo, len = max(0, seen.hi - seen.lo);
#pragma unroll 1
    for (int kt = 0; kt < 2; ++kt) {
      const uint32_t half = kt * (32 * DH * 2);
      masked_dq_tile<H, kCap, kBias>(acc, qf, dof, shift, less, k_lds + ra + half, v_lds + ra + half, k_lds + ca + half, sc, last, !whole, first + 32 * kt, len,
                                      gap - 32 * kt);
    }
  }
  __syncthreads();
  if (mine <= 0) return;
  if (slot >= 0) {                                     // a piece: [128 rows][dh] sums
    leave_sums<H>(acc, part + (((int64_t)slot * d.n_q + head) * 128 + 32 * wave) * d.dh, mine, d.dh, lane);
    return;
  }
  char* stage = reinterpret_cast<char*>(lds) + wave * RowStage<DH>::BYTES;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = acc[dt][4 * j + r] * d.grad_scale;
      RowStage<DH>::put(stage, lane, dt, j, x, false);
    }
  RowStage<DH>::flush(stage, lane, mine, d.dh, dQ + ((int64_t)row0 + 32 * wave) * d.ldq + head * d.dh, d.ldq, nullptr, 0);
}

// ---- backward: dk, dv -----------------------------------------------------------------------------------------------------------
// 32 queries x 32 keys; registers and rings as in the causal kernel.  first: index of the lane's first query relative to the first that
// sees the lane's key, of `len`; gap: distance of the lane's key from the lane's first query.
template <class H, int kCap, bool kBias>
__device__ __forceinline__ void masked_dkv_tile(f32x16 (&dk)[H::DT], f32x16 (&dv)[H::DT], const bf16x8 (&kf)[H::KS],
                                                const bf16x8 (&vf)[H::KS], const float* shift_lds, const float* delta_lds, uint32_t q_rows,
                                                uint32_t q_cols, const Scores& sc, bool last, bool masked, int first, int len, float gap, int lane) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  constexpr uint32_t kDo = Tile<DH>::ELEMS * 2;     // the dO tile follows the q tile
  typedef Tile<DH> Tl;
  constexpr int kRing = 3;
  bf16x8 f[kRing];
  f32x16 s = zero16(), dp;                 // rows = queries, column = key; dP starts at -delta, which saves the subtraction
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float4 d4 = *reinterpret_cast<const float4*>(delta_lds + 8 * j + 4 * (lane >> 5));
    dp[4 * j] = d4.x; dp[4 * j + 1] = d4.y; dp[4 * j + 2] = d4.z; dp[4 * j + 3] = d4.w;
  }
  auto fetch_rows = [&](int i) { f[i % kRing] = Tl::rows(q_rows + (i & 1) * kDo, 0, i / 2); };
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) fetch_rows(i);
#pragma unroll
  for (int i = 0; i < 2 * KS - 2; ++i) {
    if (i + kRing - 1 < 2 * KS) fetch_rows(i + kRing - 1);
    if (i % 2 == 0) s = mfma(f[i % kRing], kf[i / 2], s);
    else dp = mfma(f[i % kRing], vf[i / 2], dp);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (last) {
    s = mfma(f[(2 * KS - 2) % kRing], kf[KS - 1], s);
    dp = mfma(f[(2 * KS - 1) % kRing], vf[KS - 1], dp);
  }
  if constexpr (kCap == kWideCap) wide_scores<(KS < 8)>(sc, s, dp);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = 8 * j + 4 * (lane >> 5);
    const float4 l4 = *reinterpret_cast<const float4*>(shift_lds + row);
    const float lr[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float slack = 1.0f;
      float p = prob_of<kCap, kBias>(s[4 * j + r], sc, lr[r], gap + static_cast<float>(8 * j + r), slack);
      s[4 * j + r] = p;
      float g = p * dp[4 * j + r];
      if constexpr (kCap == kNarrowCap) g *= slack;
      dp[4 * j + r] = g;
    }
    if (j == 1 || kBias) __builtin_amdgcn_sched_barrier(0);
  }
  if (masked) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const bool ok = static_cast<uint32_t>(first + 8 * (v / 4) + v % 4) < static_cast<uint32_t>(len);
      s[v] = ok ? s[v] : 0.0f;
      dp[v] = ok ? dp[v] : 0.0f;
    }
  }
  const bf16x8 pf[2] = {pack8<0>(s), pack8<1>(s)}, df[2] = {pack8<0>(dp), pack8<1>(dp)};
  __builtin_amdgcn_sched_barrier(0);
  auto fetch_cols = [&](int i) { f[i % kRing] = Tl::cols(q_cols + (i & 1 ? 0u : kDo), 0, (i / 2) & 1, i / 4); };
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) fetch_cols(i);
#pragma unroll
  for (int i = 0; i < 4 * DT; ++i) {
    if (i + kRing - 1 < 4 * DT) fetch_cols(i + kRing - 1);
    if (i % 2 == 0) dv[i / 4] = mfma(f[i % kRing], pf[(i / 2) & 1], dv[i / 4]);
    else dk[i / 4] = mfma(f[i % kRing], df[(i / 2) & 1], dk[i / 4]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// 64 keys of a key / value head a workgroup: wavefronts 0, 2 the first 32 and 1, 3 the others; 0, 1 take the first 32 queries of every
// block of 64 and 2, 3 the others, and the two sums of a block of keys meet through LDS at the end.  All query heads of the group are walked,
// so that no sum leaves the workgroup.  K, V, dk and dv take the registers of two wavefronts a SIMD (three with heads of 64: 13 images of
// 10007 patches 153 us, with two 172).  8192 causal tokens, 16 / 8 heads of 128: 527 us (scores of deviation 1) to 620 (9), 639 capped.
template <class H, int kCap, bool kBias>
__global__ void __launch_bounds__(256, 2)
k_masked_bwd_dkv(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const bf16_t* __restrict__ dO,
                 const float* __restrict__ delta, const int* __restrict__ plan, PlanTag tag, PlanSizes z, MaskedDims d,
                 bf16_t* __restrict__ dK, bf16_t* __restrict__ dV, float* __restrict__ part) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  typedef Tile<DH> Tl;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][Tl::ELEMS];   // [stage][q, dO]
  __shared__ __attribute__((aligned(16))) float stats[2][2][kTok];         // [stage][shift, delta]
  const int item = blockIdx.x / d.n_kv, kvh = blockIdx.x % d.n_kv;
  const PlanWords w(plan, z.k_at, item, threadIdx.x & 63);
  if (!w.is(tag, true)) {
    fill_nan(dK, d.Tk, (int64_t)d.n_kv * d.dh, d.ldk);
    fill_nan(dV, d.Tk, (int64_t)d.n_kv * d.dh, d.ldv);
    return;
  }
  if (item >= w.header(kPlanKItems)) return;
  const int row0 = w.item(0), rows = w.item(1), k0 = w.item(2), q_start = w.item(3), q_len = w.item(4), off = w.item(5);
  const int prefix = w.item(6), step0 = w.item(7), steps = w.item(8) - step0, slot = w.item(9);
  const int window = tag.w[kTagWindow];
  const bool causal = tag.w[kTagFlags] & 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hi = lane >> 5;
  const int kw = wave & 1, qw = tid >> 7, heads = d.n_q / d.n_kv;   // qw as a lane's value: it chooses between registers below

  const int mine = min(32, rows - 32 * kw);            // this wavefront's keys (none: <= 0)
  const Seen sa = queries_of(k0 + 32 * kw, q_len, off, prefix, window, causal), sb = queries_of(k0 + 32 * kw + mine - 1, q_len, off, prefix, window, causal);
  const int64_t t0 = (int64_t)row0 + 32 * kw + n;

  bf16x8 kf[KS], vf[KS];     // second operands: column = key
  f32x16 dk[DT], dv[DT];     // rows = dh, column = key
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const bool on = n < mine && ks * 16 + 8 * hi < d.dh;
    const int64_t at = kvh * d.dh + ks * 16 + 8 * hi;
    kf[ks] = on ? load_frag16(K + t0 * d.ldk + at) : bf16x8{};
    vf[ks] = on ? load_frag16(V + t0 * d.ldv + at) : bf16x8{};
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dk[dt] = zero16();
    dv[dt] = zero16();
  }
  // steps: query head of the group (outer) x block of 64 queries first .. end - 1 (inner), of which the item takes a run
  const int q_lo = queries_of(k0, q_len, off, prefix, window, causal).lo, q_hi = queries_of(k0 + rows - 1, q_len, off, prefix, window, causal).hi;
  const int first = q_lo / kTok, end = q_hi > q_lo ? (q_hi + kTok - 1) / kTok : first;
  const uint32_t lds0 = lds_addr_of(lds);
  const uint32_t ra = Tl::rows_at(lane), ca = Tl::cols_at(lane);
  const bool last = uses_last<H>(d.dh);
  auto request = [&](int stage, int head, int blk) {
    const uint32_t at = lds0 + stage * (2 * Tl::ELEMS * 2);
    const int q0 = blk * kTok, me = again(tid);        // the lane's offsets are formed at every step: no registers to keep them
    const uint32_t from_q = Tl::of_lane(d.ldq, me), from_o = Tl::of_lane(d.ldo, me);
    copy_tile<DH>(Q, (int64_t)q_start + q0, q_len - q0, d.ldq, (int64_t)head * d.dh, d.dh, from_q, at, wave, tid);
    copy_tile<DH>(dO, (int64_t)q_start + q0, q_len - q0, d.ldo, (int64_t)head * d.dh, d.dh, from_o, at + Tl::ELEMS * 2, wave, tid);
    if (wave < 2)
      dma4(delta + ((int64_t)(wave == 0 ? d.n_q : 0) + head) * d.Tq + q_start + min(q0 + lane, q_len - 1),
           __builtin_amdgcn_readfirstlane(lds_addr_of(stats[stage][wave])));
  };
  int head = kvh * heads, blk = first;
  if (steps > 0) {
    head += step0 / (end - first);
    blk += step0 % (end - first);
  }
  clear_columns<H>(&lds[0][0][0], 4, d.dh, tid);
  if (steps > 0) request(0, head, blk);
  for (int it = 0; it < steps; ++it) {
    FAAR_WAIT_VMCNT(0);
    __syncthreads();
    const int i0 = blk * kTok + 32 * (wave >> 1), this_head = head;
    if (++blk == end) {
      blk = first;
      ++head;
    }
    if (it + 1 < steps) request((it + 1) & 1, head, blk);
    if (mine <= 0 || i0 >= sb.hi || i0 + 32 <= sa.lo || i0 >= q_len) continue;
    const Scores sc = scores_of(d, this_head, kBias);
    const uint32_t tile = lds0 + (it & 1) * (2 * Tl::ELEMS * 2) + (wave >> 1) * (32 * DH * 2);
    const bool whole = i0 >= sb.lo && i0 + 32 <= sa.hi;
    const int me = again(lane), key = k0 + 32 * kw + (me & 31), at = i0 + 4 * (me >> 5);
    const Seen seen = whole ? Seen{0, 0} : queries_of(key, q_len, off, prefix, window, causal);
    const float* stat = &stats[it & 1][0][32 * (wave >> 1)];
    masked_dkv_tile<H, kCap, kBias>(dk, dv, kf, vf, stat, stat + kTok, tile + ra, tile + ca, sc, last, !whole, at - seen.lo, max(0, seen.hi - seen.lo),
                                     static_cast<float>(at + off - key), lane);
  }
  // the two wavefronts of a block of keys: one hands over its dv and finishes dk, the other the reverse
  // (four values a lane at a time, side by side: no bank conflicts)
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  f32x4* give = reinterpret_cast<f32x4*>(lds) + (size_t)wave * DT * 256 + lane;
  const f32x4* take = reinterpret_cast<const f32x4*>(lds) + (size_t)(wave ^ 2) * DT * 256 + lane;
  static_assert(4 * DT * 256 * sizeof(f32x4) <= sizeof(lds), "exchange fits in the stages");
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 g;
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = qw == 0 ? dv[dt][4 * j + i] : dk[dt][4 * j + i];
      give[(dt * 4 + j) * 64] = g;
    }
  }
  __syncthreads();
  f32x16 sum[DT];
  const float k = qw == 0 && slot < 0 ? d.grad_scale : 1.0f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 r = take[(dt * 4 + j) * 64];
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[dt][4 * j + i] = ((qw == 0 ? dk[dt][4 * j + i] : dv[dt][4 * j + i]) + r[i]) * k;
    }
  }
  if (slot >= 0) {                                     // a piece: [dk, dv][64 rows][dh] sums
    leave_sums<H>(sum, part + ((((int64_t)slot * d.n_kv + kvh) * 2 + qw) * 64 + 32 * kw) * d.dh, mine, d.dh, again(lane));
    return;
  }
  __syncthreads();                                     // all has been taken: the place is free
  if (mine <= 0) return;
  char* stage = reinterpret_cast<char*>(lds) + wave * RowStage<DH>::BYTES;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x[4] = {sum[dt][4 * i], sum[dt][4 * i + 1], sum[dt][4 * i + 2], sum[dt][4 * i + 3]};
      RowStage<DH>::put(stage, lane, dt, i, x, false);
    }
  const int64_t t = (int64_t)row0 + 32 * kw, ld = qw == 0 ? d.ldk : d.ldv;
  RowStage<DH>::flush(stage, lane, mine, d.dh, (qw == 0 ? dK : dV) + t * ld + kvh * d.dh, ld, nullptr, 0);
}

// The pieces of a tile's rows, in their order: out = k * sum, of dq (kind 0, 128 rows a slot) or of dk and dv (kind 1, 64 rows of either);
// one head a workgroup.  5 to 17 us with the launch, by one round trip for the plan's words and one for the sums.
template <int kind>
__global__ void __launch_bounds__(kJoinThreads)
k_masked_join_grad(const int* __restrict__ plan, PlanTag tag, PlanSizes z, MaskedDims d, const float* __restrict__ part, bf16_t* __restrict__ A,
                   bf16_t* __restrict__ B) {
  constexpr int kSets = kind ? 2 : 1, kHeight = kind ? 64 : 128;
  const int heads = kind ? d.n_kv : d.n_q, item = blockIdx.x / heads, head = blockIdx.x % heads;
  const PlanLook<8> w(plan, z.join_at[kind], item, threadIdx.x & 63);
  if (!w.is(tag, true) || item >= w.header(kind ? kPlanKJoins : kPlanQJoins)) return;      // a wrong plan: answered by the kernel before
  const int64_t row0 = w.item(0), step = (int64_t)heads * kSets * kHeight * d.dh;
  const int rows = w.item(1), pieces = w.item(3), c8 = d.dh / 8;
  const float* first = part + ((int64_t)w.item(2) * heads + head) * kSets * kHeight * d.dh;
  for (int i = threadIdx.x; i < kSets * rows * c8; i += kJoinThreads) {
    const int set = i / (rows * c8), row = i / c8 % rows, col = i % c8 * 8;
    const float* p = first + (set * kHeight + row) * d.dh + col;
    float a[8], x[8];
    load8(p, a);
#pragma unroll 2
    for (int j = 1; j < pieces; ++j) {
      load8(p + j * step, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] += x[e];
    }
    if (set == 0)
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] *= d.grad_scale;
    const int64_t ld = kind == 0 ? d.ldq : set == 0 ? d.ldk : d.ldv;
    W8<bf16_t>::store((set == 0 ? A : B) + (row0 + row) * ld + head * d.dh + col, a);
  }
}

// ---- one token a sequence ---------------------------------------------------------------------------------------------------------
// A workgroup takes one piece of a sequence's keys for one key / value head and up to 32 of its query heads, which are the columns of
// the products: blocks of 128 keys, 32 a wavefront, two stages (four, which leave room for one workgroup a unit with heads
// of 64, are slower: 64 caches of up to 8192 keys, 8 heads, 131 -> 188 us).  The four wavefronts' sums meet through LDS; a sequence of one piece is
// done, others leave (O, maximum, denominator) of the piece in the workspace for k_masked_join.  Bound by the one pass over the cache: 96
// tokens over caches of up to 8192 keys, 8 key / value heads of 128, 1636 MB in 346 us with the join, 4.7 TB/s (a large copy: 5.0).
template <class H, int kMode>
__global__ void __launch_bounds__(256, 1)
k_masked_token(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const int* __restrict__ plan, PlanTag tag,
               PlanSizes z, MaskedDims d, bf16_t* __restrict__ O, float* __restrict__ lse, float* __restrict__ part) {
  constexpr int DH = H::DH, KS = H::KS, DT = H::DT;
  typedef Tile<DH> Tl;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][2][Tl::ELEMS];   // [stage][half of the block][k, v]
  __shared__ float ml[3][4][32];
  const int rep = d.n_q / d.n_kv, per_head = (rep + 31) / 32, cols = d.n_kv * per_head;
  const int item = blockIdx.x / cols, kvh = blockIdx.x % cols % d.n_kv, h0 = blockIdx.x % cols / d.n_kv * 32;
  const PlanWords w(plan, z.q_at, item, threadIdx.x & 63);
  if (!w.is(tag, false)) {
    fill_nan(O, d.Tq, (int64_t)d.n_q * d.dh, d.ldo);
    if (lse) fill_nan(lse, d.Tq * d.n_q);
    return;
  }
  if (item >= w.header(kPlanQItems)) return;
  const int seq = w.item(0), row0 = w.item(1), keys = w.item(2), gap0 = w.item(3), pieces = w.item(4);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hi = lane >> 5;
  const int heads = min(32, rep - h0), head = kvh * rep + h0 + min(n, heads - 1);
  const Scores sc = scores_of(d, head, kMode == kBiased || kMode == kCapped || kMode == kWide);

  MaskedState<H> st;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    st.qf[ks] = n < heads && ks * 16 + 8 * hi < d.dh ? load_frag16(Q + (int64_t)seq * d.ldq + head * d.dh + ks * 16 + 8 * hi) : bf16x8{};
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) st.oacc[dt] = zero16();
  st.mc = kMode == kBounded ? sc.ref : kLowest;
  st.l = st.lr = 0.0f;
  const int64_t kvcol = (int64_t)kvh * d.dh;
  const uint32_t lds0 = lds_addr_of(lds), ra = Tl::rows_at(lane), ca = Tl::cols_at(lane);
  const bool last = uses_last<H>(d.dh);
  const uint32_t from_k = Tl::of_lane(d.ldk, tid), from_v = Tl::of_lane(d.ldv, tid);
  constexpr uint32_t kTile = Tl::ELEMS * 2;
  auto request = [&](int blk) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = lds0 + ((blk & 1) * 2 + h) * (2 * kTile);
      const int j0 = blk * kPieceKeys + h * kTok;
      copy_tile<DH>(K, (int64_t)row0 + j0, keys - j0, d.ldk, kvcol, d.dh, from_k, at, wave, tid);
      copy_tile<DH>(V, (int64_t)row0 + j0, keys - j0, d.ldv, kvcol, d.dh, from_v, at + kTile, wave, tid);
    }
  };
  const int blocks = (keys + kPieceKeys - 1) / kPieceKeys;
  clear_columns<H>(&lds[0][0][0][0], 8, d.dh, tid);
  if (blocks > 0) request(0);
  for (int blk = 0; blk < blocks; ++blk) {
    FAAR_WAIT_VMCNT(0);
    __syncthreads();
    if (blk + 1 < blocks) request(blk + 1);
    const uint32_t k_lds = lds0 + ((blk & 1) * 2 + (wave >> 1)) * (2 * kTile), v_lds = k_lds + kTile;
    const int j0 = blk * kPieceKeys + 32 * wave;
    if (j0 >= keys) continue;
    const float gap = static_cast<float>(gap0 - j0 - 4 * hi);
    masked_block<H, kMode, 1>(st, k_lds, v_lds, ra, ca, sc, wave & 1, last, j0 + 32 > keys, j0 + 4 * hi, keys, gap, lse != nullptr);
  }
  // the wavefronts' sums on a common maximum
  const float lt = half_sum(st.l), lr = half_sum(st.lr);
  if (hi == 0) {
    ml[0][wave][n] = st.mc;
    ml[1][wave][n] = lt;
    ml[2][wave][n] = lr;
  }
  __syncthreads();                                     // and all tiles have been read
  auto joined = [&](int h, float& m, float& l, float& r) {
    m = ml[0][0][h];
    l = r = 0.0f;
#pragma unroll
    for (int i = 1; i < 4; ++i) m = fmaxf(m, ml[0][i][h]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = fast_exp2(ml[0][i][h] - m);
      l += ml[1][i][h] * f;
      r += ml[2][i][h] * f;
    }
  };
  float m, l, r;
  joined(n, m, l, r);
  const float f = fast_exp2(st.mc - m);
  float* sum = reinterpret_cast<float*>(lds);          // [wavefront][dh][32 heads]
  static_assert(4 * DH * 32 * sizeof(float) <= sizeof(lds), "sums fit in the stages");
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[(wave * DH + dt * 32 + 8 * (v / 4) + 4 * hi + v % 4) * 32 + n] = st.oacc[dt][v] * f;
  __syncthreads();
  const bool done = pieces == 1;
  if (tid < heads) {                                   // wave 0, hi 0: m and l of head n = tid
    if (!done) {
      float* o = part + ((int64_t)item * d.n_q + head) * (d.dh + kPartExtra) + d.dh;
      o[0] = m;
      o[1] = l;
      o[2] = r;
    } else if (lse) {
      lse[(int64_t)head * d.Tq + seq] = lse_of(m, l);
    }
  }
  for (int i = tid; i < heads * d.dh; i += 256) {
    const int h = i / d.dh, c = i - h * d.dh;
    float x = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) x += sum[(q * DH + c) * 32 + h];
    const int64_t hd = kvh * rep + h0 + h;
    if (!done) {
      part[((int64_t)item * d.n_q + hd) * (d.dh + kPartExtra) + c] = x;
    } else {
      float mh, lh, rh;
      joined(h, mh, lh, rh);
      O[(int64_t)seq * d.ldo + hd * d.dh + c] = static_cast<bf16_t>(f32_to_bf16(rh == 0.0f ? 0.0f : x / rh));
    }
  }
}

// The pieces of a sequence, one query head a workgroup, in their order, eight at a time: one round trip to memory brings the plan's words,
// the next all that eight pieces left.  2.8 us after one token over 700 keys, 4.8 after the 96 tokens above.
__global__ void __launch_bounds__(128)
k_masked_join(const int* __restrict__ plan, PlanTag tag, PlanSizes z, MaskedDims d, const float* __restrict__ part, bf16_t* __restrict__ O,
              float* __restrict__ lse) {
  const int seq = blockIdx.x / d.n_q, head = blockIdx.x % d.n_q;
  const PlanLook<2> w(plan, z.seq_at, seq, threadIdx.x & 63);
  const int first = w.item(0), pieces = w.item(1);
  if (!w.is(tag, false) || pieces == 1) return;        // a wrong plan: answered by the kernel before
  const int64_t step = (int64_t)d.n_q * (d.dh + kPartExtra);
  const float* p = part + first * step + head * (d.dh + kPartExtra);
  const bool on = threadIdx.x < d.dh;
  float m = kLowest, l = 0.0f, r = 0.0f, x = 0.0f;
  for (int i0 = 0; i0 < pieces; i0 += 8) {
    float mi[8], li[8], ri[8], xi[8], top = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* q = p + min(i0 + i, pieces - 1) * step;                 // the last one again, with weight 0
      mi[i] = i0 + i < pieces ? q[d.dh] : kLowest;
      li[i] = q[d.dh + 1];
      ri[i] = q[d.dh + 2];
      xi[i] = q[on ? threadIdx.x : 0];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, mi[i]);
    const float f = fast_exp2(m - top);
    l *= f;
    r *= f;
    x *= f;
    m = top;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float g = i0 + i < pieces ? fast_exp2(mi[i] - m) : 0.0f;
      l = fmaf(li[i], g, l);
      r = fmaf(ri[i], g, r);
      x = fmaf(xi[i], g, x);
    }
  }
  if (on) O[(int64_t)seq * d.ldo + head * d.dh + threadIdx.x] = static_cast<bf16_t>(f32_to_bf16(r == 0.0f ? 0.0f : x / r));
  if (lse && threadIdx.x == 0) lse[(int64_t)head * d.Tq + seq] = lse_of(m, l);
}

}  // namespace

PlanSizes attention_plan_sizes(int64_t n_seq, int64_t Tq, int64_t Tk, int64_t n_q, int64_t n_kv, bool single) {
  PlanSizes z{};
  z.q_at = 16;
  if (single) {
    const int64_t cols = n_kv * ((n_q / n_kv + 31) / 32);
    // pieces: about 512 workgroups; small caches in one piece each, since joining costs as much as walking four blocks of
    // keys.  Pieces with their join against whole, on the device: 512 rows, 16 heads of 128 7.0 + 2.8 against 9.2 us and 8 heads of 64
    // 5.8 + 2.9 against 6.8; but 700 rows, 8 heads of 64 5.5 + 3.2 against 10.3
    z.target = Tk <= kSmallCaches ? 0 : static_cast<int>((512 + cols - 1) / cols);
    z.max_q = n_seq + z.target;
    z.seq_at = static_cast<int>(z.q_at + kItemWords * z.max_q);
    z.words = z.seq_at + 2 * n_seq;
    return z;
  }
  // Tiles in pieces: where the rows make fewer workgroups than the device holds a time and a half (768 of 128 queries; 1024 of the
  // shorter ones of 64 keys).  There are then at most as many pieces beyond one a tile as fill it, and none longer than what each of those
  // has to do on average.  With enough tiles the most expensive first are balance enough: 24 documents in 8192 tokens, 16 / 8 heads of
  // 128, dq 80 us without, 79 with pieces, dk and dv 75 and 84, and each list to join costs its launch.  With few they are most of the speed, in us
  // without / with: 1 x 10612 tokens, 2 heads of 128, forward 261 / 109, dq 394 / 168, dk and dv 308 / 200; 3 sequences in 8192, 16 heads of
  // 64 on one, dk and dv 1080 / 194.  None where no tile is as long as two pieces.
  const int64_t tq = Tq / 128 + n_seq, tk = Tk / kTok + n_seq;
  const int64_t long_q = (Tk + kTok - 1) / kTok, long_k = n_q / n_kv * ((Tq + kTok - 1) / kTok);
  auto extra = [](int64_t full_tiles, int64_t enough, int64_t slots, int64_t heads, int64_t tiles, int64_t longest) {
    if (full_tiles * heads >= enough) return 0;
    return static_cast<int>(std::min((slots + heads - 1) / heads, tiles * ((longest + kLeastPiece - 1) / kLeastPiece - 1)));
  };
  z.extra_q = extra(Tq / 128, 768, 512, n_q, tq, long_q);
  z.extra_k = extra(Tk / kTok, 1024, 1024, n_kv, tk, long_k);
  z.max_q = tq + z.extra_q;
  z.max_k = tk + z.extra_k;
  int64_t at = z.q_at + kItemWords * z.max_q;
  auto take = [&](int64_t words) {
    const int64_t r = at;
    at += words;
    return static_cast<int>(r);
  };
  z.k_at = take(kItemWords * z.max_k);
  z.join_at[0] = take(8 * std::max(1, z.extra_q));
  z.join_at[1] = take(8 * std::max(1, z.extra_k));
  z.words = at;
  return z;
}

// float32 sums of pieces: of the forward; of the backward behind delta, first dq's, then in the same place those of dk and dv
int64_t masked_fwd_floats(const PlanSizes& z, const MaskedDims& d, bool single) {
  if (single) return z.max_q * d.n_q * (d.dh + kPartExtra);
  return (int64_t)2 * z.extra_q * d.n_q * 128 * (d.dh + kPartExtra);
}
int64_t masked_bwd_floats(const PlanSizes& z, const MaskedDims& d) {
  return round_up((int64_t)2 * d.n_q * d.Tq, 64) + std::max((int64_t)2 * z.extra_q * d.n_q * 128 * d.dh, (int64_t)2 * z.extra_k * d.n_kv * 128 * d.dh);
}

hipError_t launch_attention_plan(const int* q_start, const int* q_len, const int* k_start, const int* k_len, const int* prefix, const PlanTag& tag,
                                 const PlanSizes& z, int* plan, hipStream_t st) {
  hipLaunchKernelGGL(k_attention_plan, dim3(1), dim3(kPlanThreads), 0, st, q_start, q_len, k_start, k_len, prefix, tag, z, plan);
  return hipGetLastError();
}

hipError_t launch_masked_fwd(const bf16_t* Q, const bf16_t* K, const bf16_t* V, const int* plan, const PlanTag& tag, const PlanSizes& z,
                             const MaskedDims& d, bool single, bf16_t* O, float* lse, uint8_t* o_low, float* part, hipStream_t st) {
  // A capped score is at most a = cap log2(e): with exponents from 2^-110 (reference a - 110 at least, so that none is lost) to
  // 2^40 (a <= 75) sums of 2^20 of them with values of up to 2^60 stay in range, and at the low end, where all of a row's scores are -cap,
  // products end at 2^-149, 2^-39 of v's unit; so no running maximum is needed (8192 causal tokens, 16 / 8 heads of 128: 390 us
  // without, 406 with).
  const int mode = d.cap_a > kNarrow ? kWide : d.cap_a > 0.0f ? (!d.slopes && d.cap_a <= 75.0f ? kBounded : kCapped) : d.slopes ? kBiased : kPlain;
  const int rep = d.n_q / d.n_kv;
  const int64_t cols = (int64_t)d.n_kv * ((rep + 31) / 32);
  const dim3 grid(static_cast<unsigned>(single ? z.max_q * cols : z.max_q * d.n_q));
#define FAAR_MF2(H, M)                                                                                                              \
  do {                                                                                                                              \
    if (single) hipLaunchKernelGGL((k_masked_token<H, M>), grid, dim3(256), 0, st, Q, K, V, plan, tag, z, d, O, lse, part);         \
    else hipLaunchKernelGGL((k_masked_fwd<H, M>), grid, dim3(256), 0, st, Q, K, V, plan, tag, z, d, O, lse, o_low, part);           \
  } while (0)
  // heads of 65 .. 96 as 96 rather than 128: 13 images of 10007 patches, heads of 80, forward 121 / 136 us, dq 151 / 168, dk and dv 221 / 247
#define FAAR_MF(M) \
  do { if (d.dh <= 64) FAAR_MF2(Heads64, M); else if (d.dh <= 96) FAAR_MF2(Heads96, M); else FAAR_MF2(Heads128, M); } while (0)
  switch (mode) {
    case kPlain: FAAR_MF(kPlain); break;
    case kBiased: FAAR_MF(kBiased); break;
    case kBounded: FAAR_MF(kBounded); break;
    case kCapped: FAAR_MF(kCapped); break;
    default: FAAR_MF(kWide); break;
  }
#undef FAAR_MF
#undef FAAR_MF2
  if (hipError_t e = hipGetLastError()) return e;
  if (!single && z.extra_q > 0)
    hipLaunchKernelGGL(k_masked_join_fwd, dim3(static_cast<unsigned>(z.extra_q * d.n_q)), dim3(kJoinThreads), 0, st, plan, tag, z, d, part, O, lse, o_low);
  if (single && z.target > 0)
    hipLaunchKernelGGL(k_masked_join, dim3(static_cast<unsigned>(d.Tq * d.n_q)), dim3(128), 0, st, plan, tag, z, d, part, O, lse);
  return hipGetLastError();
}

hipError_t launch_masked_bwd(const bf16_t* dO, const bf16_t* Q, const bf16_t* K, const bf16_t* V, const bf16_t* O, const uint8_t* o_low, const float* lse,
                             const int* plan, const PlanTag& tag, const PlanSizes& z, const MaskedDims& d, float* ws, bf16_t* dQ, bf16_t* dK,
                             bf16_t* dV, hipStream_t st) {
  float *delta = ws, *part = ws + round_up(2 * d.n_q * d.Tq, 64);
  const dim3 gq(static_cast<unsigned>(z.max_q * d.n_q)), gk(static_cast<unsigned>(z.max_k * d.n_kv));
#define FAAR_MB2(H, C, B)                                                                                                               \
  do {                                                                                                                                  \
    hipLaunchKernelGGL((k_masked_bwd_dq<H, C, B>), gq, dim3(256), 0, st, Q, K, V, dO, O, o_low, lse, plan, tag, z, d, delta, dQ, part); \
    if (z.extra_q > 0)                                                                                                                  \
      hipLaunchKernelGGL(k_masked_join_grad<0>, dim3(static_cast<unsigned>(z.extra_q * d.n_q)), dim3(kJoinThreads), 0, st, plan, tag, z, d, part, dQ, dQ); \
    hipLaunchKernelGGL((k_masked_bwd_dkv<H, C, B>), gk, dim3(256), 0, st, Q, K, V, dO, delta, plan, tag, z, d, dK, dV, part);           \
  } while (0)
#define FAAR_MB(C, B) \
  do { if (d.dh <= 64) FAAR_MB2(Heads64, C, B); else if (d.dh <= 96) FAAR_MB2(Heads96, C, B); else FAAR_MB2(Heads128, C, B); } while (0)
  if (d.cap_a > kNarrow) FAAR_MB(kWideCap, true);
  else if (d.cap_a > 0.0f) { if (d.slopes) FAAR_MB(kNarrowCap, true); else FAAR_MB(kNarrowCap, false); }
  else                     { if (d.slopes) FAAR_MB(kNoCap, true); else FAAR_MB(kNoCap, false); }
#undef FAAR_MB
#undef FAAR_MB2
  if (hipError_t e = hipGetLastError()) return e;
  if (z.extra_k > 0)
    hipLaunchKernelGGL(k_masked_join_grad<1>, dim3(static_cast<unsigned>(z.extra_k * d.n_kv)), dim3(kJoinThreads), 0, st, plan, tag, z, d, part, dK, dV);
  return hipGetLastError();
}

}  // namespace faar
