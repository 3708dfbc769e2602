// Device code of the kernels that recompute attention probabilities (backward pass, key weights): unpadded tiles in LDS
// and matrix operands with the head dimension in half-split order.
#pragma once

#include "lazy_attn_device.h"

namespace lazy {
namespace {

// Tiles in LDS: rows of D bf16, unpadded (a row of 64 or 32 banks), whose 16-byte chunks are permuted: chunk c of row r
// lies at place c ^ swizzle(r).  Two kinds of reads are conflict free then: rows by 16 lanes of consecutive rows (one
// chunk each: swizzle takes as many values as there are chunks over the rows that share banks) and transposing reads,
// whose passes cover four chunks 4 b .. 4 b + 3 of four consecutive rows (rows that share banks differ in the bits of
// swizzle that select b).
template <int D>
__device__ __forceinline__ int swizzle(int r) {
  return D == 128 ? ((r & 3) << 2 | (r >> 2 & 3)) : ((r >> 1 & 1) << 2 | (r >> 2 & 3));
}
template <int D>
__device__ __forceinline__ int tile_at(int row, int chunk) {
  return row * D + 8 * (chunk ^ swizzle<D>(row));
}
// x, in a way that the compiler does not see through: what is computed from it is computed where it stands, not kept in
// registers across a loop.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A lane's operands of 32x32x16 products from a tile.  row: elements 16 k + 8 (lane / 32) .. + 7 of row row0 + lane % 32.
// column: transposed, element column 32 db + lane % 32 of rows row0 + {0..3, 8..11} + 4 (lane / 32), the rows that
// registers 8 j .. 8 j + 7 of an accumulator hold for this lane half (row0 a multiple of 16; row's of 32).  Steps only
// flip bits of the chunk index, so every address is one exclusive or away from two.
template <int D>
struct TileOperands {
  int ra, ca;
  __device__ explicit TileOperands(int lane) {
    const int i = lane & 15;
    ra = 2 * tile_at<D>(lane & 31, lane >> 5);
    ca = 2 * (tile_at<D>(4 * (lane >> 5) + (i >> 2), 2 * (lane >> 4 & 1) + ((i & 3) >> 1)) + 4 * (i & 1));
  }
  __device__ __forceinline__ bf16x8 row(const uint16_t* tile, int row0, int k) const {
    return as_bf16x8(*reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(tile) + 2 * D * row0 + (ra ^ 32 * k)));
  }
  __device__ __forceinline__ bf16x8 column(const uint16_t* tile, int row0, int db) const {
    const char* at = reinterpret_cast<const char*>(tile) + 2 * D * row0;
    const u32x2 lo = tr_read(reinterpret_cast<const uint16_t*>(at + (ca ^ 64 * db)));
    const u32x2 hi = tr_read(reinterpret_cast<const uint16_t*>(at + 16 * D + (ca ^ 32 ^ 64 * db)));
    return as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
  }
};

// Rows of 16-byte chunks copied to a tile in LDS without passing through registers: lane l of a wave writes the 16 bytes
// at 16 l from a uniform base, so the tile's permutation of chunks is made by the lanes' source addresses.
__device__ __forceinline__ void copy_async(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)from,
                                   (__attribute__((address_space(3))) uint32_t*)to, 16, 0, 0);
}
// The same, four bytes a lane.
__device__ __forceinline__ void copy_async4(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)from,
                                   (__attribute__((address_space(3))) uint32_t*)to, 4, 0, 0);
}
// Every copy and LDS access so far has ended; nothing moves across.
__device__ __forceinline__ void wait_copies() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// Every LDS access so far has ended; no memory access moves across.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Packed row -> token: row / G by multiplication (total_q * G * G < 2^32, checked by the planner).
__device__ __forceinline__ int token_of(int row, uint32_t magic) { return magic ? (int)__umulhi(row, magic) : row; }

// Eight pairs t0 .. t0 + 7 of a vector in global memory: first elements lo, second elements hi.
template <int D, bool IL>
__device__ __forceinline__ void load_pairs(const uint16_t* v, int t0, u32x4& lo, u32x4& hi) {
  if (IL) {
    const u32x4* src = reinterpret_cast<const u32x4*>(v + 2 * t0);
    const u32x4 a = src[0], b = src[1];
    deinterleave8(a, b, lo, hi);
  } else {
    lo = *reinterpret_cast<const u32x4*>(v + t0);
    hi = *reinterpret_cast<const u32x4*>(v + D / 2 + t0);
  }
}
__device__ __forceinline__ float element(const u32x4& v, int e) { return (e & 1) ? bf_hi(v[e >> 1]) : bf_lo(v[e >> 1]); }
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  return u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}
// Eight fp32 values as the sum of two bf16 ones each: rounded, and what is left, rounded.  The sum is within 2^-16 of the
// value (relative), against 2^-8 for the first alone.  (Cutting off the lower half instead of rounding costs as many
// instructions and makes every rest twice as large and of its value's sign.)
__device__ __forceinline__ void split8(const float (&v)[8], u32x4& hi, u32x4& lo) {
  hi = pack8(v);
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = v[e] - element(hi, e);
  lo = pack8(rest);
}
template <int D, bool IL>
__device__ __forceinline__ void store_pairs(uint16_t* v, int t0, const float (&lo)[8], const float (&hi)[8]) {
  if (IL) {
    const float a[8] = {lo[0], hi[0], lo[1], hi[1], lo[2], hi[2], lo[3], hi[3]};
    const float b[8] = {lo[4], hi[4], lo[5], hi[5], lo[6], hi[6], lo[7], hi[7]};
    reinterpret_cast<u32x4*>(v + 2 * t0)[0] = pack8(a);
    reinterpret_cast<u32x4*>(v + 2 * t0)[1] = pack8(b);
  } else {
    *reinterpret_cast<u32x4*>(v + t0) = pack8(lo);
    *reinterpret_cast<u32x4*>(v + D / 2 + t0) = pack8(hi);
  }
}

// ALiBi's slopes and the log-sum-exps enter the kernels of these scores as they are, not times log2 e: bias and log-sum-exp
// may each be far larger than their difference, which is rounded once (fmaf) and then scaled.
constexpr float lse_scale(int km) { return km == kKeysAlibi ? 1.f : kLog2e; }
template <class Args>
__device__ __forceinline__ float natural_slope(const Args& a, int h) {
  return a.inv_freq ? a.inv_freq[h] : exp2f(-8.0f * (float)(h + 1) / (float)a.hq);
}
__device__ __forceinline__ float biased(float slope, int distance, float nlse) {
  return fmaf(slope, (float)distance, nlse) * kLog2e;
}

// Rotations per position of pair t, in revolutions: from the caller's table, or as the host worked them out.
template <class Args>
__device__ __forceinline__ double revolutions(const Args& a, int t) {
  return a.inv_freq ? (double)a.inv_freq[t] * kInvTwoPi : a.rev[t];
}

// Angles of positions 0 .. 31, which a 32-key block's keys add to the position of its first: (cos, sin) of [32][D/2] pairs
// by kAngleBlocks workgroups of 256.
template <int D>
constexpr int kAngleBlocks = kAngleRows * (D / 2) / 256;
template <int D, class Args>
__device__ __forceinline__ void angle_rows(const Args& a, int block) {
  const int e = block * 256 + threadIdx.x;
  reinterpret_cast<float2*>(a.ws_angles)[e] = rope_cs(e / (D / 2), revolutions(a, e % (D / 2)));
}

// The operands of a 32-key block.  Lane: key `row` of its 64-key tile, elements 16 s + 8 h2 .. + 7 of operand s; its pairs
// lie in operand s + D / 32.  First as they are stored, all loads in flight together (interleaved pairs: 16 elements).
template <int D, bool IL>
__device__ __forceinline__ void load_keys(const uint16_t* krow, int h2, u32x4 (&kf)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const int t0 = 16 * s + 8 * h2;
    kf[s] = *reinterpret_cast<const u32x4*>(krow + (IL ? 2 * t0 : t0));
    kf[s + D / 32] = *reinterpret_cast<const u32x4*>(krow + (IL ? 2 * t0 + 8 : D / 2 + t0));
  }
}
// Then rotated.  base: (cos, sin) of the tile's position (local-position keys: of their record's), in LDS; rows(t): those
// of the lane's key within the tile, for pairs t and t + 1.
template <int D, int KM, bool IL, class Rows>
__device__ __forceinline__ void rotate_pairs(const u32x4& a, const u32x4& b, int t0, const float2* base, Rows rows,
                                             float (&yl)[8], float (&yh)[8]) {
  u32x4 lo = a, hi = b;
  if (IL) deinterleave8(a, b, lo, hi);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    if (KM == kKeysLocal) {
      rotate_by(element(lo, e), element(hi, e), base[t0 + e], yl[e], yh[e]);
      rotate_by(element(lo, e + 1), element(hi, e + 1), base[t0 + e + 1], yl[e + 1], yh[e + 1]);
    } else {
      const f32x4 r = rows(t0 + e);
      rotate_pair(element(lo, e), element(hi, e), base[t0 + e], make_float2(r[0], r[1]), yl[e], yh[e]);
      rotate_pair(element(lo, e + 1), element(hi, e + 1), base[t0 + e + 1], make_float2(r[2], r[3]), yl[e + 1], yh[e + 1]);
    }
  }
}
// As two bf16 parts.
template <int D, int KM, bool IL, class Rows>
__device__ __forceinline__ void rotate_keys_split(u32x4 (&kh)[D / 16], u32x4 (&kl)[D / 16], int h2, const float2* base,
                                                  Rows rows) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    float yl[8], yh[8];
    rotate_pairs<D, KM, IL>(kh[s], kh[s + D / 32], 16 * s + 8 * h2, base, rows, yl, yh);
    split8(yl, kh[s], kl[s]);
    split8(yh, kh[s + D / 32], kl[s + D / 32]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace
}  // namespace lazy
