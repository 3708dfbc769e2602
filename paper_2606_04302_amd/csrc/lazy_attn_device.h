// Device code that the kernels of this library share: bf16 and wave helpers, rotation angles, the walk over a request's
// records, and the layouts of tiles in LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "lazy_attn_internal.h"

namespace lazy {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a8 __attribute__((ext_vector_type(4), aligned(8)));  // in a caller's record table

constexpr int kThreads = 256;
constexpr int kSub = 64;  // keys of one loader sub-tile; tile row 0 of a sub-tile is a multiple of 64 in its chunk
constexpr int kPad = 8;   // bf16 elements of padding per LDS row
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLog2e = 1.4426950408889634f;
// The softmax reference max only moves when a tile's max exceeds it by more than this (log2 units): unnormalised
// probabilities stay below 2^8, far inside fp32 and bf16 range, and the O accumulator is rescaled rarely.
constexpr float kRescaleSlack = 8.0f;
constexpr float kRescaleBound = 256.0f;  // 2^kRescaleSlack
constexpr double kInvTwoPi = 0.15915494309189533577;

static_assert(kPrefillTileKeys == kSub, "prefill tiles are one loader sub-tile");

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// A value that is the same in every lane of the wave, marked as such.  The compiler cannot prove it for values
// derived from threadIdx (the wave index) or computed with the vector integer-division expansion; without the mark
// the chunk-table walk that depends on them runs as divergent vector code, its record loads become vector loads,
// and their waits drain the vector-memory queue that holds the next tile's prefetched K / V.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Inclusive prefix sum over the 64 lanes of a wave (all lanes active), with DPP lane moves instead of LDS
// permutes: shifts by 1, 2, 4, 8 within each 16-lane row (lanes shifted in from outside the row read 0), then the
// last lane of row 0 is added to row 1 and that of row 2 to row 3 (row_bcast:15), then the last lane of row 1
// (the total of rows 0-1) to rows 2 and 3 (row_bcast:31).  Rows left out by the row mask keep their value.
__device__ __forceinline__ int wave_incl_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15, rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31, rows 2 and 3
  return x;
}
// Reductions over lane pairs (l, l ^ 32) with v_permlane32_swap (one VALU op, no LDS round trip).  Swapping a
// register with itself yields x[l % 32] in one result and x[l % 32 + 32] in the other, in every lane, so both
// lanes of a pair combine the same two values in the same order.
__device__ __forceinline__ float xor32_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xor32_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// acc + (lo + hi) of a packed bf16 pair (v_dot2c_f32_bf16 with weights 1): the softmax denominator is summed over
// the same bf16-rounded probabilities that enter the P V product.
__device__ __forceinline__ float add_pair(uint32_t pair, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, acc,
                                         false);
}

// theta_t / (2 pi): RoPE frequency of pair t in revolutions per position (original RoPE: base^(-2t/D), evaluated as
// exp2(-(2t/D) log2(base)) with log2(base) from the host, far cheaper than a double pow; RoPE variants pass their own
// table, Sec. 3.5).
__device__ __forceinline__ double theta_rev(int t, int d, double log2_base, const float* inv_freq) {
  const double th = inv_freq ? (double)inv_freq[t] : exp2(-2.0 * (double)t / (double)d * log2_base);
  return th * kInvTwoPi;
}

// (cos, sin) of the angle p * theta for theta given in revolutions: the product and its fractional part in fp64
// (exact range reduction for any position below 2^24), then the hardware sine and cosine, which take the angle in
// revolutions (v_sin_f32 / v_cos_f32; on [0, 1) within 1.3e-7 of the exact values, measured on an MI355X against
// fp64, about twice the error of a libm-style sincospi at a tenth of the instructions).
__device__ __forceinline__ float2 rope_cs(int p, double rev) {
  const float r = (float)__builtin_amdgcn_fract((double)p * rev);
  return make_float2(__builtin_amdgcn_cosf(r), __builtin_amdgcn_sinf(r));
}

// Rotate one pair (x1, x2) = (k[t], k[t + D/2]) by the angle base + delta, given (cos, sin) of each part.
// Written with explicit fmaf so that every kernel that rotates keys rounds identically.
__device__ __forceinline__ void rotate_pair(float x1, float x2, float2 cb, float2 cd, float& y1, float& y2) {
  const float c = fmaf(cb.x, cd.x, -(cb.y * cd.y));
  const float s = fmaf(cb.y, cd.x, cb.x * cd.y);
  y1 = fmaf(x1, c, -(x2 * s));
  y2 = fmaf(x1, s, x2 * c);
}

// Rotate one pair by a single angle given its (cos, sin): the one rotation of a local-position key by its record's
// offset.  Same fmaf form in every kernel that uses it.
__device__ __forceinline__ void rotate_by(float x1, float x2, float2 cs, float& y1, float& y2) {
  y1 = fmaf(x1, cs.x, -(x2 * cs.y));
  y2 = fmaf(x1, cs.y, x2 * cs.x);
}

// Key handling of a kernel instance: keys already encoded at their positions (the plain kernels of the
// materialise-then-attend baseline), NoPE keys rotated at pos_offset + j, or local-position keys (stored encoded at
// j) rotated by the record's pos_offset.
constexpr int kKeysPlain = 0, kKeysNope = 1, kKeysLocal = 2;
// Score-space positions (ALiBi): keys and queries are used as stored and slope_h (k_pos - q_pos) is added to every
// scaled score (Sec. 3.5 "Score-space positional methods").
constexpr int kKeysAlibi = 3;

// ALiBi slope of query head h: table[h], or 2^(-8 (h+1) / Hq); returned divided by the softmax scale (times
// log2 e over scale_log2), so that adding slope' (k_pos - q_pos) to the raw dot product adds the bias to the scaled
// score.
__device__ __forceinline__ float alibi_slope(int h, int hq, const float* table, float scale_log2) {
  const float sl = table ? table[h] : exp2f(-8.0f * (float)(h + 1) / (float)hq);
  return sl * 1.4426950408889634f / scale_log2;
}
// Bit 2 of a kernel's key-mode argument selects the interleaved pairing (pairs (2t, 2t+1)).  Interleaved RoPE on
// (q, k) is the half-split rotation of (P q, P k) for the permutation P: 2t -> t, 2t+1 -> t + D/2 (V unchanged), so
// the kernels only change their Q and K loads: 16 consecutive elements are split into the pairs' first and second
// halves, the layout a half-split load produces, and everything after the load is shared.
constexpr int kInterleaved = 4;
constexpr int keys_of(int km) { return km & 3; }
constexpr bool interleaved_of(int km) { return (km & kInterleaved) != 0; }
// Bit 3 of a decode kernel's key-mode argument: K and V are read with non-temporal loads (LAZY_CACHE_STREAM).
constexpr int kStreamKV = 8;
constexpr bool stream_of(int km) { return (km & kStreamKV) != 0; }

// 16 bf16 = pairs t0..t0+7 of an interleaved vector (w0: pairs t0..t0+3, one pair per 32-bit word, first element
// in the low half; w1: pairs t0+4..t0+7) -> the first elements (lo) and second elements (hi) in pair order.
__device__ __forceinline__ void deinterleave8(u32x4 w0, u32x4 w1, u32x4& lo, u32x4& hi) {
  lo = u32x4{(w0[0] & 0xffffu) | (w0[1] << 16), (w0[2] & 0xffffu) | (w0[3] << 16), (w1[0] & 0xffffu) | (w1[1] << 16),
             (w1[2] & 0xffffu) | (w1[3] << 16)};
  hi = u32x4{(w0[0] >> 16) | (w0[1] & 0xffff0000u), (w0[2] >> 16) | (w0[3] & 0xffff0000u),
             (w1[0] >> 16) | (w1[1] & 0xffff0000u), (w1[2] >> 16) | (w1[3] & 0xffff0000u)};
}
// Four pairs: 8 bf16 of an interleaved vector -> first and second elements.
__device__ __forceinline__ void deinterleave4(u32x4 w, u32x2& lo, u32x2& hi) {
  lo = u32x2{(w[0] & 0xffffu) | (w[1] << 16), (w[2] & 0xffffu) | (w[3] << 16)};
  hi = u32x2{(w[0] >> 16) | (w[1] & 0xffff0000u), (w[2] >> 16) | (w[3] & 0xffff0000u)};
}

// Rotate a query pair at position p (accurate angle per pair).
__device__ __forceinline__ void rotate_q_pair(float x1, float x2, int p, double rev, float& y1, float& y2) {
  const float2 cs = rope_cs(p, rev);
  y1 = fmaf(x1, cs.x, -(x2 * cs.y));
  y2 = fmaf(x1, cs.y, x2 * cs.x);
}

struct Rec {
  int64_t koff, voff;
  int len, pos, kst, vst;
};

// Read-only tables are read through the constant address space: uniform loads from it become scalar loads, whose
// waits (lgkmcnt) do not drain the vector-memory queue that holds the next tile's prefetched K / V.
template <typename T>
using cptr = const T __attribute__((address_space(4)))*;
template <typename T>
__device__ __forceinline__ cptr<T> as_const(const T* p) {
  return (cptr<T>)p;
}

__device__ __forceinline__ Rec load_rec(cptr<lazy_chunk_t> c) {
  Rec r;
  r.koff = c->k_offset;
  r.voff = c->v_offset;
  r.len = c->len;
  r.pos = c->pos_offset;
  r.kst = c->k_stride;
  r.vst = c->v_stride;
  return r;
}

// Walks the key tiles of one request that belong to one KV split: tiles never straddle chunks; the request's
// tiles (chunk after chunk, TK keys each, the last one of a chunk possibly partial) are numbered and split
// evenly.  With the causal rule, tiles whose first key lies after the last query of the workgroup are skipped.
template <int TK>
struct TileIter {
  cptr<lazy_chunk_t> recs;
  int i, end, j0, left;
  Rec cur, nxt;  // records i and i + 1 (nxt only while i + 1 < end): the next record is always loaded ahead

  // The tile counts are taken one record per lane, 64 records at a time, with a wave-wide prefix sum, so that a long
  // chunk table costs a few parallel loads rather than a chain of dependent ones.  Must be called by whole waves
  // with wave-uniform arguments; every member ends up wave-uniform.
  //
  // The loads of the first 256 records come first and on their own (first_block), so that a caller can issue other
  // loads while they are in flight: record c0 + lane whole (the record holding the split's first tile and the one
  // after it then come from a lane instead of one more dependent load), and the lengths of records
  // c0 + 64 (u + 1) + lane.  Indexes past the table's end read its last record and are ignored afterwards, so no
  // load sits behind a per-lane branch.
  struct First {
    lazy_chunk_t mine;
    int len[3];
  };
  __device__ static First first_block(const lazy_chunk_t* table, int c0, int c1) {
    First f = {};
    if (c1 > c0) {
      const int k = c0 + (threadIdx.x & 63);
      f.mine = table[min(k, c1 - 1)];
#pragma unroll
      for (int u = 0; u < 3; ++u) f.len[u] = table[min(k + 64 * (u + 1), c1 - 1)].len;
    }
    return f;
  }
  __device__ void init(const lazy_chunk_t* table, int c0, int c1, int split, int splits) {
    init(table, c0, c1, split, splits, first_block(table, c0, c1));
  }
  __device__ void init(const lazy_chunk_t* table, int c0, int c1, int split, int splits, const First& first) {
    recs = as_const(table);
    if (!locate(table, c0, c1, split, splits, first)) return;
    const int f = i - c0;
    if (f < 64) {
      cur = lane_rec(first.mine, f);
      if (i + 1 < end) nxt = f + 1 < 64 ? lane_rec(first.mine, f + 1) : load_rec(recs + i + 1);
    } else {
      cur = load_rec(recs + i);
      if (i + 1 < end) nxt = load_rec(recs + i + 1);
    }
  }
  // Number and place of the split's tiles: left, i and j0; false if the split holds none.
  __device__ bool locate(const lazy_chunk_t* table, int c0, int c1, int split, int splits, const First& first) {
    end = c1;
    const int lane = threadIdx.x & 63;
    const lazy_chunk_t& mine = first.mine;
    // Pass 1: the request's tile count, four blocks of 64 records at a time; the first four blocks' counts stay in
    // registers for pass 2.
    int ntiles = 0, ntb[4];
    for (int k0 = c0; k0 < c1; k0 += 256) {
      int nt[4], sum = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = k0 + 64 * u + lane;
        const int len = k0 != c0 ? (k < c1 ? table[k].len : 0) : u == 0 ? mine.len : first.len[u - 1];
        nt[u] = k < c1 ? (len + TK - 1) / TK : 0;
        if (k0 == c0) ntb[u] = nt[u];
        sum += nt[u];
      }
      ntiles += __builtin_amdgcn_readlane(wave_incl_scan(sum), 63);
    }
    const int lo = (int)((int64_t)ntiles * split / splits);
    const int hi = (int)((int64_t)ntiles * (split + 1) / splits);
    left = hi - lo;
    i = c1;
    j0 = 0;
    if (left <= 0) return false;
    // Pass 2: the record holding tile lo, the first whose inclusive tile count exceeds lo.
    int acc = 0;
    for (int k0 = c0; k0 < c1; k0 += 64) {
      const int k = k0 + lane;
      const int b = (k0 - c0) >> 6;
      const int nt = b < 4 ? (b == 0 ? ntb[0] : b == 1 ? ntb[1] : b == 2 ? ntb[2] : ntb[3])
                           : (k < c1 ? (table[k].len + TK - 1) / TK : 0);
      const int incl = acc + wave_incl_scan(nt);
      const uint64_t hit = __ballot(k < c1 && incl > lo);
      if (hit) {
        const int f = __builtin_ctzll(hit);
        i = k0 + f;
        j0 = (lo - __builtin_amdgcn_readlane(incl - nt, f)) * TK;
        break;
      }
      acc = __builtin_amdgcn_readlane(incl, 63);
    }
    return true;
  }
  // Lane f's record as a wave-uniform value.
  __device__ static Rec lane_rec(const lazy_chunk_t& r, int f) {
    Rec x;
    x.koff = ((int64_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)r.k_offset >> 32), f) << 32) |
             (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)r.k_offset, f);
    x.voff = ((int64_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)r.v_offset >> 32), f) << 32) |
             (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)r.v_offset, f);
    x.len = __builtin_amdgcn_readlane(r.len, f);
    x.pos = __builtin_amdgcn_readlane(r.pos_offset, f);
    x.kst = __builtin_amdgcn_readlane(r.k_stride, f);
    x.vst = __builtin_amdgcn_readlane(r.v_stride, f);
    return x;
  }
  __device__ void step() {
    --left;
    j0 += TK;
    // Zero-length records own no tile, so while tiles are left a record with keys lies ahead.
    while (left > 0 && j0 >= cur.len) {
      ++i;
      j0 = 0;
      cur = nxt;
      if (i + 1 < end) nxt = load_rec(recs + i + 1);
    }
  }
  // Move to the next tile that some query of the workgroup can see (the current one included).
  __device__ bool seek(bool causal, int qmax) {
    while (left > 0) {
      if (!causal || cur.pos + j0 <= qmax) return true;
      step();
    }
    return false;
  }
};

// Angles: the rotation of key j of a chunk (position pos + j) uses one decomposition everywhere (lazy kernels and
// the materialising copy), so every path produces bit-identical rotated keys:
//     angle(pos + j) = base(pos + 32 * floor(j / 32)) + row(j mod 32)
// with cos/sin of each part from rope_cs and one angle addition (rotate_pair).
constexpr int kAngleRows = 32;

// LDS layout constants of a 64-key prefill tile.  Bank-conflict notes: gfx950 LDS has 64 banks of 4 bytes and
// serves a 16-byte read for 16 lanes per pass (8-byte reads: 32 lanes per pass; writes: 8 lanes per pass, half
// the read rate); a pattern is conflict free when the lanes of one pass that read distinct addresses cover
// distinct banks.
//  - K tile rows are D + 8 elements apart (a 4-bank shift per row, so 16 consecutive rows of one 16-byte column
//    tile the 64 banks); the 16-byte blocks of a row are permuted by kblk_t().
//  - The V tile is row-major (key, dimension) with rows D + 32 elements apart (a 16-bank shift per row): the
//    transposing reads (ds_read_b64_tr_b16: 32 lanes read 4 rows x 64 bytes per pass) hit 4 disjoint 16-bank
//    groups.  With rows D + 16 apart they conflict two ways.
//  - cos/sin rows interleave (c, s) with a 4-float gap after every 32 pairs (cs_idx), and the per-row table has a
//    row stride of 8 (mod 64) floats for D = 128 and 4 for D = 64: the 16-byte reads of the loader threads of
//    one pass (4 or 8 threads per key row) hit distinct banks.
template <int D>
struct TileLayout {
  static constexpr int KLD = D + kPad;                    // K tile: [64][KLD], head dimension in virtual order
  static constexpr int VLD = D + 32;                      // V tile: [64][VLD], natural layout
  static constexpr int CSW = D + 4 * ((D / 2 - 1) / 32);  // floats per cos/sin row: (c, s) of pair t at cs_idx(t)
  static constexpr int CSD_LD = CSW + 4;                  // row stride of the per-row table
};

// Transposing LDS read (gfx950 ds_read_b64_tr_b16).  Within each group of 16 lanes, lane i supplies the address
// of 4 consecutive 16-bit elements M[i][0..3]; lane j receives M[4e + j/4][j%4] for e = 0..3.  With lane i pointing
// at row (base + i/4) and column (4 * (i%4)) of a row-major tile, lane j gets column j of rows base..base+3, which is
// an MFMA operand fragment of four consecutive keys for one dimension.
typedef short i16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2 tr_read(const uint16_t* p) {
  const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
  return __builtin_bit_cast(u32x2, v);
}
template <int D>
__device__ __forceinline__ int cs_idx(int t) { return 2 * t + 4 * (t / 32); }

__device__ __forceinline__ const uint16_t* k_ptr(const uint16_t* pool, const Rec& r, int g, int j0, int d) {
  return pool + r.koff + ((int64_t)g * r.kst + j0) * d;
}
__device__ __forceinline__ const uint16_t* v_ptr(const uint16_t* pool, const Rec& r, int g, int j0, int d) {
  return pool + r.voff + ((int64_t)g * r.vst + j0) * d;
}

// Base tables of a 64-key tile whose first key sits at position b0: [0] for rows 0..31, [1] for rows 32..63.
// For local-position keys b0 is the record offset and both halves get its angles.
template <int D, bool LOCAL>
__device__ __forceinline__ void prefill_base(float* csb2, const double* freq, int tid, int b0) {
  if (tid < D) {
    const int h = tid / (D / 2), t = tid % (D / 2);
    *reinterpret_cast<float2*>(csb2 + h * TileLayout<D>::CSW + cs_idx<D>(t)) =
        rope_cs(LOCAL ? b0 : b0 + kAngleRows * h, freq[t]);
  }
}

}  // namespace
}  // namespace lazy
