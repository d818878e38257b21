// What the attention kernels share: matrix-core operands in registers, asynchronous copies into LDS, and tiles of 64 tokens in
// LDS that are read by rows and, transposed, by columns.
#pragma once
#include "faar_internal.h"

namespace faar {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTok = 64;       // tokens per LDS tile

union Frag {
  bf16x8 v;
  uint4 q;
  uint32_t w[4];
};

__device__ __forceinline__ bf16x8 load_frag16(const bf16_t* p) {   // 8 consecutive bf16
  Frag f;
  f.q = *reinterpret_cast<const uint4*>(p);
  return f.v;
}
// accumulator registers 8 t .. 8 t + 7 of a tile -> the second operand of a 16-token step
template <int T>
__device__ __forceinline__ bf16x8 pack8(const f32x16& a) {
  Frag f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f.w[i] = pack_bf16x2(a[8 * T + 2 * i], a[8 * T + 2 * i + 1]);
  return f.v;
}
__device__ __forceinline__ f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}
// the values of lane i and lane i ^ 32, in either order (v_permlane32_swap: a vector instruction, no LDS round trip)
__device__ __forceinline__ void both_halves(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float x) {
  float a, b;
  both_halves(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float half_sum(float x) {
  float a, b;
  both_halves(x, a, b);
  return a + b;
}
__device__ __forceinline__ void store4_bf16(bf16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}

// 2^x by the hardware instruction alone: results below 2^-126 may flush to zero, and above 2^128 they are infinite (under a cap, of which the
// reciprocal is taken; exponents of probabilities stay within a few units of zero, or 40 against a fixed reference)
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// 16 bytes (4 in the second form) per lane from global memory straight into LDS at lds_addr + 16 * lane (4 * lane), lds_addr
// wave-uniform.  Inline assembly: the compiler does not see the LDS write, so completion is tracked by hand (wait_vmcnt, then
// the workgroup barrier); its own wait counts for ordinary loads stay sufficient, since memory operations return in order.
__device__ __forceinline__ void dma16(const void* base, uint32_t lane_offset, uint32_t lds_addr) {   // base wave-uniform
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(lane_offset), "s"(base)
               : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* gptr, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_addr), "v"(gptr) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr_of(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}
#define FAAR_WAIT_VMCNT(N) __builtin_amdgcn_s_waitcnt(0x0F70 | ((N)&0xF) | (((N) >> 4) << 14))

// A [64 tokens][dh] tile of a token-major tensor in LDS, rows un-padded.  The 16-byte chunks of a row are stored XOR-permuted
// by a key of the row so that both kinds of read spread over the 64 banks, which serve 16 lanes of a 16-byte row read or 32 of an
// 8-byte transposing read at a time: the 16 rows of the one fall on 16 distinct chunk positions, and the 8 32-byte segments of the
// other (4 tokens x 2 groups of 16 columns) on the 8 bank groups once each.  dh = 128: a row is one turn of the banks, and its bits
// 0, 1, 2, 3 go to bits 2, 3, 1, 0 of the chunk (bits 1..3: which 32-byte segment, bit 1 the group of 16 columns); dh = 64: two rows
// to a turn, bits 1, 2, 3 to bits 2, 1, 0.  (With row bits in order, which keeps 64 lanes apart but not each 32, every transposing
// read took twice the cycles.)
template <int DH>
struct Tile {
  static constexpr int CPR = DH / 8;                  // 16-byte chunks per row
  static constexpr int COPIES = kTok * CPR / 256;     // copies per thread
  static constexpr int ELEMS = kTok * DH;

  static __device__ __forceinline__ int key(int row) {
    return (DH == 128 ? 4 * (row & 3) : 2 * (row & 2)) | ((row >> 1) & 2) | ((row >> 3) & 1);
  }
  // rows row0 .. row0+63, columns col0 .. col0+dh-1, global -> LDS without passing through registers: chunk i = tid + 256 j of
  // the tile lands at byte 16 i.  A pass of the workgroup covers 2048 / dh rows, a divisor of 32, and starts at a row whose key
  // is 0, so one lane offset (of_lane) serves every pass.  `valid` rows are there (32, or 64 and more): the passes beyond them
  // repeat the first one, and callers mask what comes of those rows.
  static __device__ __forceinline__ uint32_t of_lane(int64_t ld, int tid) {
    const int row = tid / CPR;
    return static_cast<uint32_t>(row * ld * 2) + ((tid % CPR) ^ key(row)) * 16;
  }
  static __device__ __forceinline__ void copy(const bf16_t* __restrict__ src, int64_t row0, int valid, int64_t ld, int64_t col0,
                                              uint32_t lane_offset, uint32_t tile, int wave) {
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
      const int row = j * (256 / CPR);
      dma16(src + (row0 + (row < valid ? row : 0)) * ld + col0, lane_offset,
            __builtin_amdgcn_readfirstlane(tile + 4096u * j + 1024u * wave));
    }
  }
  // LDS byte addresses of a lane's reads: everything but the compile-time parts, which are added, or XORed into the chunk bits
  // (a row is a power of two long: the bits above it never change).  rows: row lane % 32, the 8 values at 8 (lane / 32).  cols:
  // within 16 lanes, lane r supplies the address of 4 columns of one token and receives one column of 4 tokens; the tokens come
  // in the order a lane holds them in an accumulator tile: 4 (lane / 32) + 0..3, then 8 further on (chunk bit 0 flips, key).
  static __device__ __forceinline__ uint32_t rows_at(int lane) {
    return (lane & 31) * (DH * 2) + ((lane >> 5) ^ key(lane & 31)) * 16;
  }
  static __device__ __forceinline__ uint32_t cols_at(int lane) {
    const int r = lane & 15, row = 4 * (lane >> 5) + (r >> 2);   // token of a 16-token step
    return row * (DH * 2) + ((2 * ((lane >> 4) & 1) + ((r & 3) >> 1)) ^ key(row)) * 16 + (r & 1) * 8;
  }
  // rows 32 half .. +31 x 16 of dh (step ks) of the tile whose LDS address is already in `at` (an aligned tile: a plain sum, but
  // the compiler does not know; formed per step and made opaque, it leaves the constant parts to the instruction's offset field)
  static __device__ __forceinline__ bf16x8 rows(uint32_t at, int half, int ks) {
    typedef __attribute__((address_space(3))) const bf16x8* ptr;
    uint32_t x = at ^ (32u * ks);
    asm("" : "+v"(x));
    return *reinterpret_cast<ptr>(x + half * (32 * DH * 2));
  }
  // dh rows 32 dt .. +31 x 16 tokens (step st of the 32 tokens `half`)
  static __device__ __forceinline__ bf16x8 cols(uint32_t at, int half, int st, int dt) {
    typedef __attribute__((address_space(3))) s16x4* ptr;
    uint32_t x = at ^ (64u * dt), y = at ^ (64u * dt + 16u);
    asm("" : "+v"(x), "+v"(y));
    const uint32_t off = (half * 32 + st * 16) * (DH * 2);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(x + off));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ptr>(y + off + 8 * (DH * 2)));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, v);
  }
};

}  // namespace
}  // namespace faar
