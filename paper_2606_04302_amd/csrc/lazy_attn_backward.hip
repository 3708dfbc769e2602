// Backward pass of the prefill attention for gfx950: gradients of the queries and of the stored keys and values.
//
// Two to four launches.  (1) prepare_rows: queries rotated to their positions and packed by KV head (row = token * G +
// head in group), dO packed alike, and two numbers a row, -lse log2 e and -delta.  (2) grad_kv: dk and dv, one tile of
// the store at a time.  (3) grad_q: dq, one row tile and key split at a time.  (4) finish: partial dq of requests in
// several key splits summed, turned back and rounded, and the same for tiles whose uses were cut into parts; only where
// there are any. (2) and (3) are one launch, grad_all, unless there is much work for 256 rows a workgroup
// (kMostTogether).  The probabilities are recomputed in (2) and in (3): seven products of the two kernels against five
// if dq were summed over key tiles with atomics, whose order would change results from call to call.
//
// Precision: rotated queries and keys, P and dS are each the sum of two bf16 numbers (split8, 2^-17), and a product of
// two of them is three products, first x first and the two mixed ones; V, dO and ALiBi's queries and keys are exact as
// they are. One part each, 2^-9 a term, is no error of 2^-9: where a handful of keys holds nearly all of a row's
// weight, elements of a gradient are far smaller than their terms and far above the tensor's root mean square (3 rows
// over 28000 ALiBi keys: elements wrong by 0.84 of the larger of themselves and that mean; scores of standard deviation
// 4: 0.03 to 1.4, and 1% in the 2-norm).  Two parts leave the rounding of the result (0.0039, 0.0017 in the 2-norm) and
// make sixteen of seven products: 16 ragged requests 3.9 ms instead of 1.85, 8 requests with 64 rows a chunk 0.40
// instead of 0.21.
//
// Rotations: scores are products of keys and queries rotated to their absolute positions, as in the forward pass.  In
// every tile in LDS and in every operand the head dimension is in half-split order, so that the pair (t, t + D/2) of a
// row or of an accumulator column lies in one lane; interleaved pairs are split when they are loaded and joined when
// they are stored.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lazy_attn_backward.h"
#include "lazy_attn_device.h"
#include "lazy_attn_internal.h"
#include "lazy_attn_tiles.h"

namespace lazy {
namespace {

constexpr int kMaxBlockTokens = 16;

// Queries rotated, in two parts, packed by KV head; row constants.  One workgroup a block of tokens, D / 16 threads a row.
// Bound by memory: 5015 tokens of 32 heads of 64 22 us for 123 MB (5.6 TB/s, part of it from the caches).
template <int D, bool IL>
__global__ __launch_bounds__(256) void prepare_rows(GradArgs a) {
  __shared__ float2 cs[kMaxBlockTokens][D / 2];
  const GradBlock b = a.blocks[blockIdx.x];
  if (a.rotate_q) {
    for (int e = threadIdx.x; e < b.tokens * (D / 2); e += 256)
      cs[e / (D / 2)][e % (D / 2)] = rope_cs(b.t0 + e / (D / 2) + b.pos_shift, revolutions(a, e % (D / 2)));
    __syncthreads();
  }
  constexpr int TPR = D / 16;
  const int t0 = 8 * (threadIdx.x % TPR);
  for (int row = threadIdx.x / TPR; row < b.tokens * a.hq; row += 256 / TPR) {
    const int tok = row / a.hq, h = row % a.hq;
    const int64_t src = (int64_t)(b.t0 + tok) * a.hq + h;
    const int64_t dst = (int64_t)(h / a.group) * a.rows + (int64_t)(b.t0 + tok) * a.group + h % a.group;
    u32x4 lo, hi;
    load_pairs<D, IL>(a.q + src * D, t0, lo, hi);
    const float lse = a.lse[src];
    const bool dead = lse == -INFINITY;  // a row that sees no key: zeros, whatever stands in it
    if (dead) lo = hi = u32x4{};
    float yl[8], yh[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      yl[e] = element(lo, e);
      yh[e] = element(hi, e);
      if (a.rotate_q) rotate_by(element(lo, e), element(hi, e), cs[tok][t0 + e], yl[e], yh[e]);
    }
    u32x4 rest;
    uint16_t* const second = a.ws_q + (a.hkv * a.rows + dst) * D;
    split8(yl, lo, rest);
    if (a.parts > 1) *reinterpret_cast<u32x4*>(second + t0) = rest;
    split8(yh, hi, rest);
    if (a.parts > 1) *reinterpret_cast<u32x4*>(second + D / 2 + t0) = rest;
    *reinterpret_cast<u32x4*>(a.ws_q + dst * D + t0) = lo;
    *reinterpret_cast<u32x4*>(a.ws_q + dst * D + D / 2 + t0) = hi;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      u32x4 x = *reinterpret_cast<const u32x4*>(a.dout + src * D + 2 * t0 + 8 * k);
      if (dead) x = u32x4{};
      *reinterpret_cast<u32x4*>(a.ws_do + dst * D + 2 * t0 + 8 * k) = x;
      const u32x4 y = *reinterpret_cast<const u32x4*>(a.out + src * D + 2 * t0 + 8 * k);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(element(x, e), element(y, e), sum);
    }
#pragma unroll
    for (int m = 1; m < TPR; m <<= 1) sum += __shfl_xor(sum, m, 64);
    if (t0 == 0) {
      if (a.dlse) sum -= a.dlse[src];
      a.ws_info[dst] = dead ? -INFINITY : -lse * a.lse_scale;  // exp2(0 - inf) = 0
      a.ws_info[a.hkv * a.rows + dst] = dead ? 0.f : -sum;
    }
  }
}

// Key and value gradients.  A workgroup owns a tile of two 64-key halves, each of its four waves 32 keys: K (rotated,
// both parts) stays in registers and V in LDS, as the right-hand operands of S = Q K^T and dP = dO V^T, whose
// accumulators have a key in every lane and 32 query rows in registers and lane halves; P and dS leave them, in two
// parts, as the right-hand operands of dV^T += dO^T P and dK^T += Q^T dS without any exchange between lanes.  S, dV, dP
// and dK follow each other, so that besides K and the sums only one or two of them are in registers.  Q and dO come
// through LDS, 32 rows at a time, read by rows for S and dP and transposed for dV and dK.  -delta is dP's initial
// value.  dK is kept in the rotated frame of the use at hand and turned on when the next use has another position.
//
// Two waves a SIMD hide each other's latencies, and one workgroup's products the other's copies: with a second buffer
// for the next 32 rows, head_dim 128 would leave one workgroup a CU (64 with one and three workgroups: kMostTogether).
// Bound by the products: 16 ragged requests, 2.2 TFLOP of nine products 2.1 ms (1050 TFLOP/s, 86% of the large library
// product's rate); 8 requests of 64 rows a chunk 211 us, where a tile has 8 to 24 steps and its loads, rotations and
// results are a third.

// A use as a wave's half of the tile sees it, and a step over it.
struct Use {
  int row_begin, row_end, pos_shift, full_from, pos, record_pos, key_begin, key_end;
};
struct Step {
  Use use;
  int row0;
};
// 32 query rows in LDS: both parts of Q, dO, and -lse (times log2 e but for ALiBi), then -delta.
template <int D, bool ROT>
struct RowTiles {
  uint16_t q[(ROT ? 2 : 1) * kGradRows * D] __attribute__((aligned(16)));
  uint16_t d[kGradRows * D] __attribute__((aligned(16)));
  float in[2 * kGradRows] __attribute__((aligned(16)));
};
template <int D, int KMI>
struct KeySmem {
  static constexpr int KM = keys_of(KMI);
  // A key's angle is that of its block of eight keys, a table of each wave's, and that of its place in the block, a table
  // of the workgroup's (rows four banks apart).  Loaded from memory, in the operands' layout, they kept the CU's address
  // units busy for 4096 cycles a use, and again at the end (64 rows a chunk: 148 us instead of 138).
  static constexpr int RLD = D / 2 + 2;
  RowTiles<D, KM != kKeysAlibi> rows;
  uint16_t v[4][32 * D] __attribute__((aligned(16)));  // a wave's V operands, then its results
  int rpos[4][kGradRows] __attribute__((aligned(16)));
  float rslope[4][KM == kKeysAlibi ? kGradRows : 4] __attribute__((aligned(16)));
  float2 turn[4][KM == kKeysAlibi ? 2 : KM == kKeysLocal ? RLD : 4 * RLD] __attribute__((aligned(16)));
  float2 place[KM == kKeysNope ? 8 * RLD : 2] __attribute__((aligned(16)));
};
template <int D, int KMI>
__device__ __forceinline__ void key_gradients(const GradArgs& a, int id, KeySmem<D, KMI>& sm) {
  constexpr int KM = keys_of(KMI);
  constexpr bool ALIBI = KM == kKeysAlibi, ROT = !ALIBI, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  constexpr int C = D / 8;  // chunks of a row
  constexpr int COPIES = kGradRows * C / 256;
  constexpr int RLD = KeySmem<D, KMI>::RLD;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h2 = lane >> 5, g = id % a.hkv;
  const int hf = wave >> 1, k32 = 32 * (wave & 1), key = k32 + (lane & 31);
  const cptr<GradTile> tile = as_const(a.tiles) + id / a.hkv;
  const struct {
    int64_t k_off, v_off;
    int kst, vst, keys;
  } t = {tile->half[hf].k_off, tile->half[hf].v_off, tile->half[hf].kst, tile->half[hf].vst, tile->half[hf].keys};
  const int seg_begin = tile->seg_begin, seg_end = tile->seg_end, part = tile->part;
  const bool active = k32 < t.keys;  // a wave without keys only helps to copy
  int* const rpos = sm.rpos[wave];
  float* const rslope = sm.rslope[wave];
  float2* const turn = sm.turn[wave];
  float2* const place = sm.place;
  uint16_t* const tv = sm.v[wave];
  const double rev = ROT ? revolutions(a, lane % (D / 2)) : 0.0;
  const auto block_angles = [&](int pos, int step) {  // of pos, pos + step, ..: one for local-position keys
    const int l = again(lane);
#pragma unroll
    for (int e = 0; e < (LOCAL ? D / 2 : 2 * D); e += 64)
      if (!LOCAL || l < D / 2)
        turn[(e + l) / (D / 2) * RLD + l % (D / 2)] = rope_cs(pos + (e + l) / (D / 2) * step, rev);
    wait_reads();
  };
  const float2* const own_turn = turn + (LOCAL ? 0 : (lane & 31) / 8 * RLD);
  const float2* const own_place = place + (LOCAL ? 0 : (lane & 7) * RLD);
  if (KM == kKeysNope) {
    static_assert(256 % (D / 2) == 0, "a thread's entries share one pair");
    for (int e = threadIdx.x; e < 8 * (D / 2); e += 256) place[e / (D / 2) * RLD + e % (D / 2)] = rope_cs(e / (D / 2), rev);
    __syncthreads();
  }
  const int own_key = min(key, t.keys - 1);  // lanes past the last key repeat it; their columns are not stored

  u32x4 kh[D / 16], kl[D / 16];
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) dk[db] = dv[db] = f32x16{};
  const uint16_t* krow = a.k_pool + t.k_off + ((int64_t)g * t.kst + own_key) * D;
  if (active) {
    const uint16_t* v = a.v_pool + t.v_off + (int64_t)g * t.vst * D;
#pragma unroll
    for (int i = 0; i < 32 * C / 64; ++i) {
      const int row = (64 * i + lane) / C, chunk = (64 * i + lane) % C ^ swizzle<D>(row);
      copy_async(v + min(k32 + row, t.keys - 1) * D + 8 * chunk, tv + 512 * i);
    }
  }
  const uint16_t* qbase = a.ws_q + (int64_t)g * a.rows * D;
  const int64_t second = a.hkv * a.rows * D;  // from a query's first part to its second
  const uint16_t* dbase = a.ws_do + (int64_t)g * a.rows * D;
  const float* ibase = a.ws_info + (int64_t)g * a.rows;
  int frame = 0;  // position by which dk is rotated (NoPE: that of the half's key 0)
  bool first = true;

  const auto load_use = [&](int i) {
    const cptr<GradSeg> u = as_const(a.segs) + i;
    const cptr<GradSeg::Half> h = &u->half[hf];
    return Use{u->row_begin, u->row_end, u->pos_shift, u->full_from, h->pos, h->record_pos, h->key_begin, h->key_end};
  };

  RowTiles<D, ROT>& tiles = sm.rows;
  const auto fetch = [&](const Step& step) {
    const int row0 = step.row0, most = step.use.row_end - 1 - row0;  // rows past the use's end repeat its last one
    const uint16_t* q = qbase + (int64_t)row0 * D;
    const uint16_t* d = dbase + (int64_t)row0 * D;
    const int e0 = again(threadIdx.x);
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const int row = (256 * i + e0) / C, chunk = ((256 * i + e0) % C) ^ swizzle<D>(row);
      const int off = min(row, most) * D + 8 * chunk;
      copy_async(q + off, tiles.q + 2048 * i + 512 * wave);
      if (ROT) copy_async(q + second + off, tiles.q + kGradRows * D + 2048 * i + 512 * wave);
      copy_async(d + off, tiles.d + 2048 * i + 512 * wave);
    }
    if (wave == 0)
      copy_async4(ibase + (lane & 32 ? a.hkv * a.rows : 0) + row0 + min(lane & 31, most), tiles.in);
  };

  const auto compute = [&](const Step& step) {
    const uint16_t *const tq = tiles.q, *const tq2 = tiles.q + kGradRows * D, *const td = tiles.d;
    const float* const in = tiles.in;
    const Use& seg = step.use;
    const int row0 = step.row0, rows = min(kGradRows, seg.row_end - row0), pos = seg.pos;
    if (row0 == seg.row_begin) {  // a new use: its keys, and dk turned on to its frame
      const int l = again(lane);
      const int here = LOCAL ? seg.record_pos : pos;
      load_keys<D, IL>(krow, l >> 5, kh);
      if (ROT) {
        if (!first && here != frame) {
          if (l < D / 2) turn[l] = rope_cs(here - frame, rev);
          wait_reads();
#pragma unroll
          for (int db = 0; db < D / 64; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float x1 = dk[db][i], x2 = dk[db + D / 64][i];
              float y1, y2;
              rotate_by(x1, x2, turn[32 * db + 8 * (i >> 2) + 4 * h2 + (i & 3)], y1, y2);
              dk[db][i] = y1;
              dk[db + D / 64][i] = y2;
              if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
          wait_reads();
        }
        block_angles(LOCAL ? here : here + k32, 8);
      }
      if (ROT)
        rotate_keys_split<D, KM, IL>(kh, kl, l >> 5, own_turn,
                                     [&](int t) { return *reinterpret_cast<const f32x4*>(own_place + t); });
      frame = here;
      first = false;
    }
    const bool masked = row0 < seg.full_from || rows < kGradRows;
    if (ALIBI || masked) {
      if (lane < kGradRows) {
        const int src = row0 + lane, tok = token_of(src, a.group_magic);
        rpos[lane] = lane >= rows ? INT32_MIN : a.causal || ALIBI ? tok + seg.pos_shift : INT32_MAX - 1;
        if (ALIBI) rslope[lane] = natural_slope(a, g * a.group + src - tok * a.group);
      }
      wait_reads();
    }

    const TileOperands<D> op(again(lane));
    // Operands are read one step ahead of their products, and the scheduler is fenced at every step: the reads in flight
    // hide their latency without taking more registers than there are.
    f32x16 s = f32x16{};
    bf16x8 fq[2], fl[2], fd[2], fv[2];
    fq[0] = op.row(tq, 0, 0);
    if (ROT) fl[0] = op.row(tq2, 0, 0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if (k + 1 < D / 16) {
        fq[(k + 1) & 1] = op.row(tq, 0, k + 1);
        if (ROT) fl[(k + 1) & 1] = op.row(tq2, 0, k + 1);
      }
      if (ROT) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fl[k & 1], as_bf16x8(kh[k]), s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[k & 1], as_bf16x8(kl[k]), s, 0, 0, 0);
      }
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[k & 1], as_bf16x8(kh[k]), s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    fd[0] = op.column(td, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(in + 8 * q4 + 4 * h2);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 8 * q4 + 4 * h2 + e;
        const float y = ALIBI ? biased(rslope[row], pos + key - rpos[row], x[e]) : x[e];
        s[4 * q4 + e] = fast_exp2(fmaf(s[4 * q4 + e], a.scale_log2, y));
      }
    }
    if (masked) {
      // Keys that the use does not have lie past every row.
      const bool used = key >= seg.key_begin && key < seg.key_end;
      const int p = !used ? INT32_MAX : a.causal ? pos + key : 0;
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int4 last = *reinterpret_cast<const int4*>(rpos + 8 * q4 + 4 * h2);
        const int at[4] = {last.x, last.y, last.z, last.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * q4 + e] = p <= at[e] ? s[4 * q4 + e] : 0.f;
      }
    }
    // Eight rows of x in two parts, the right-hand operands of the products over rows.
    const auto parts = [](const f32x16& x, int k, u32x4& hi, u32x4& lo) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[8 * k + e];
      split8(y, hi, lo);
    };
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      u32x4 hi, lo;
      parts(s, k, hi, lo);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int at = k * (D / 32) + db, ahead = at + 1;
        if (ahead < 2 * (D / 32)) fd[ahead & 1] = op.column(td, 16 * (ahead / (D / 32)), ahead % (D / 32));
        dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[at & 1], as_bf16x8(lo), dv[db], 0, 0, 0);
        dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[at & 1], as_bf16x8(hi), dv[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    f32x16 dp;
    fd[0] = op.row(td, 0, 0);
    fv[0] = op.row(tv, 0, 0);
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(in + kGradRows + 8 * q4 + 4 * h2);
#pragma unroll
      for (int e = 0; e < 4; ++e) dp[4 * q4 + e] = y[e];
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if (k + 1 < D / 16) {
        fd[(k + 1) & 1] = op.row(td, 0, k + 1);
        fv[(k + 1) & 1] = op.row(tv, 0, k + 1);
      }
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[k & 1], fv[k & 1], dp, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    fq[0] = op.column(tq, 0, 0);
    if (ROT) fl[0] = op.column(tq2, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (masked) {  // hidden pairs: 0, also where dp has overflowed
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] = s[i] > 0.f ? dp[i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= dp[i];
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      u32x4 hi, lo;
      parts(s, k, hi, lo);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int at = k * (D / 32) + db, ahead = at + 1;
        if (ahead < 2 * (D / 32)) {
          fq[ahead & 1] = op.column(tq, 16 * (ahead / (D / 32)), ahead % (D / 32));
          if (ROT) fl[ahead & 1] = op.column(tq2, 16 * (ahead / (D / 32)), ahead % (D / 32));
        }
        if (ROT) dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fl[at & 1], as_bf16x8(hi), dk[db], 0, 0, 0);
        dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[at & 1], as_bf16x8(lo), dk[db], 0, 0, 0);
        dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[at & 1], as_bf16x8(hi), dk[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };
  if (seg_begin < seg_end) {
    int si = seg_begin;
    Step now{load_use(si), 0}, next;
    now.row0 = now.use.row_begin;
    Use ahead = load_use(min(si + 1, seg_end - 1));
    const auto advance = [&] {  // next: the step after now; false at the end
      next = now;
      next.row0 += kGradRows;
      if (next.row0 < now.use.row_end) return true;
      if (++si >= seg_end) return false;
      next = {ahead, ahead.row_begin};
      ahead = load_use(min(si + 1, seg_end - 1));
      return true;
    };
    fetch(now);
    while (true) {
      const bool more = advance();
      wait_copies();
      __syncthreads();
      if (active) compute(now);
      if (!more) break;
      now = next;
      __syncthreads();
      fetch(now);
    }
  }
  wait_copies();
  if (!active) return;

  // Scaled, and turned back to the frame in which the key is stored.
  const float scale = a.scale_log2 * kLn2;
  if (ROT) block_angles(LOCAL ? -frame : -(frame + k32), -8);
#pragma unroll
  for (int db = 0; db < D / 64; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int pair = 32 * db + 8 * q4 + 4 * h2;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * q4 + e;
        float x1 = dk[db][i] * scale, x2 = dk[db + D / 64][i] * scale;
        if (ROT) {
          float2 cs = LOCAL ? make_float2(1.f, 0.f) : own_place[pair + e];
          cs.y = -cs.y;
          rotate_pair(x1, x2, own_turn[pair + e], cs, x1, x2);
        }
        dk[db][i] = x1;
        dk[db + D / 64][i] = x2;
      }
    }
  if (part >= 0) {
    float* out = a.ws_parts + ((((int64_t)part * a.hkv + g) * kGradHalves + hf) * 2 * kGradTileKeys + key) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int col = 32 * db + 8 * q4 + 4 * h2;
        *reinterpret_cast<f32x4*>(out + col) =
            f32x4{dk[db][4 * q4], dk[db][4 * q4 + 1], dk[db][4 * q4 + 2], dk[db][4 * q4 + 3]};
        *reinterpret_cast<f32x4*>(out + kGradTileKeys * D + col) =
            f32x4{dv[db][4 * q4], dv[db][4 * q4 + 1], dv[db][4 * q4 + 2], dv[db][4 * q4 + 3]};
      }
    return;
  }
  // Through LDS, so that whole rows are written: a lane has neighbouring elements of one key, four at a time.
  uint16_t* const stage = tv;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int col = 32 * db + 8 * q4 + 4 * h2;
        const f32x16& x = which ? dk[db] : dv[db];
        if (!IL || !which) {
          *reinterpret_cast<u32x2*>(stage + tile_at<D>(lane & 31, col / 8) + col % 8) =
              u32x2{pack2(x[4 * q4], x[4 * q4 + 1]), pack2(x[4 * q4 + 2], x[4 * q4 + 3])};
        } else if (db < D / 64) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = pack2(dk[db][4 * q4 + e], dk[db + D / 64][4 * q4 + e]);
          *reinterpret_cast<u32x4*>(stage + tile_at<D>(lane & 31, col / 4)) = w;
        }
      }
    wait_reads();
    uint16_t* out = which ? a.dk_pool + t.k_off + ((int64_t)g * t.kst + k32) * D
                          : a.dv_pool + t.v_off + ((int64_t)g * t.vst + k32) * D;
#pragma unroll
    for (int i = 0; i < 32 * C / 64; ++i) {
      const int row = (64 * i + lane) / C, chunk = (64 * i + lane) % C;
      if (k32 + row < t.keys)
        *reinterpret_cast<u32x4*>(out + row * D + 8 * chunk) =
            *reinterpret_cast<const u32x4*>(stage + tile_at<D>(row, chunk));
    }
    wait_reads();
  }
}
template <int D, int KMI>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void grad_kv(GradArgs a) {
  __shared__ KeySmem<D, KMI> sm;
  key_gradients<D, KMI>(a, blockIdx.x, sm);
}

// Loads a 64-key tile of K and V for a workgroup of NT threads, NT / 64 a key row, rotates the keys and writes both to
// LDS in two parts (unpadded tiles, pairs in half-split order).  The angles of the 32 rows are read from LDS for every
// tile: the eight-wave kernel has no registers for them.
template <int D, int KMI, int NT>
struct TileLoader {
  using S = TileLayout<D>;
  static constexpr int KM = keys_of(KMI);
  static constexpr bool ROT = KM == kKeysNope || KM == kKeysLocal, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  static constexpr int TPR = NT / kSub, PP = D / (2 * TPR), NV = PP / 8, VC = kSub * (D / 8) / NT;
  static_assert(PP % 8 == 0 && VC * TPR == D / 8);
  u32x4 ka[NV], kb[NV], vr[VC];  // raw pairs: first and second halves (interleaved: 16 elements as stored)
  int row, part;
  __device__ void init(int t) {
    row = t / TPR;
    part = t % TPR;
  }
  // Rows past the record's end repeat its last key; their products are masked.
  __device__ void fetch(const uint16_t* k, const uint16_t* v, int nvalid) {
    const int r = min(row, nvalid - 1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int t0 = part * PP + 8 * i;
      const uint16_t* src = k + r * D;
      ka[i] = *reinterpret_cast<const u32x4*>(src + (IL ? 2 * t0 : t0));
      kb[i] = *reinterpret_cast<const u32x4*>(src + (IL ? 2 * t0 + 8 : D / 2 + t0));
    }
#pragma unroll
    for (int i = 0; i < VC; ++i) vr[i] = *reinterpret_cast<const u32x4*>(v + r * D + 8 * (part + TPR * i));
  }
  __device__ void store(uint16_t* tk, uint16_t* tk2, uint16_t* tv, const float* cb2, const float* csd) {
    const float* cb = cb2 + (row / kAngleRows) * S::CSW;
    const float* cd = csd + (row & (kAngleRows - 1)) * S::CSD_LD;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int t0 = part * PP + 8 * i;
      u32x4 lo = ka[i], hi = kb[i];
      if (IL) deinterleave8(ka[i], kb[i], lo, hi);
      if (ROT) {
        float yl[8], yh[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int ci = cs_idx<D>(t0 + e);
          if (LOCAL) {
            rotate_by(element(lo, e), element(hi, e), *reinterpret_cast<const float2*>(cb + ci), yl[e], yh[e]);
          } else {
            rotate_pair(element(lo, e), element(hi, e), *reinterpret_cast<const float2*>(cb + ci),
                        *reinterpret_cast<const float2*>(cd + ci), yl[e], yh[e]);
          }
        }
        u32x4 rest;
        split8(yl, lo, rest);
        *reinterpret_cast<u32x4*>(tk2 + tile_at<D>(row, t0 / 8)) = rest;
        split8(yh, hi, rest);
        *reinterpret_cast<u32x4*>(tk2 + tile_at<D>(row, D / 16 + t0 / 8)) = rest;
      }
      *reinterpret_cast<u32x4*>(tk + tile_at<D>(row, t0 / 8)) = lo;
      *reinterpret_cast<u32x4*>(tk + tile_at<D>(row, D / 16 + t0 / 8)) = hi;
    }
#pragma unroll
    for (int i = 0; i < VC; ++i) *reinterpret_cast<u32x4*>(tv + tile_at<D>(row, part + TPR * i)) = vr[i];
  }
};

template <int D, int KMI, int NBUF>
struct GradQSmem {
  using S = TileLayout<D>;
  static constexpr bool ROT = keys_of(KMI) != kKeysAlibi;
  uint16_t k[NBUF][(ROT ? 2 : 1) * kSub * D] __attribute__((aligned(16)));  // both parts
  uint16_t v[NBUF][kSub * D] __attribute__((aligned(16)));
  float csd[kAngleRows * S::CSD_LD] __attribute__((aligned(16)));
  float csb[2][2][S::CSW] __attribute__((aligned(16)));
  double freq[D / 2];
};

// dS of one 64-key tile for a wave's 32 query rows, and its product: S^T = K Q^T and dP^T = V dO^T have a query row in
// every lane; dS^T leaves them as the right-hand operand of dQ^T += K^T dS^T.
template <int D, bool ALIBI>
__device__ __forceinline__ void grad_tile(const uint16_t* tk, const uint16_t* tv, int lane, const bf16x8 (&qf)[D / 16],
                                          const bf16x8 (&ql)[D / 16], const bf16x8 (&df)[D / 16],
                                          f32x16 (&dq)[D / 32], float scale_log2, float nl, float nd, float slope,
                                          int qpos, int b0, int nvalid, int qmin, int causal) {
  constexpr bool ROT = !ALIBI;
  const int h2 = lane >> 5;
  const bool masked = nvalid < kSub || (causal && b0 + kSub - 1 > qmin);
  const TileOperands<D> op(again(lane));
  const uint16_t* const tk2 = tk + kSub * D;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    f32x16 s = f32x16{}, dp;
    __builtin_amdgcn_s_setprio(1);
    // Operands one step ahead of their products.
    bf16x8 fk[2], fl[2], fv[2];
    fk[0] = op.row(tk, 32 * kb, 0);
    if (ROT) fl[0] = op.row(tk2, 32 * kb, 0);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if (k + 1 < D / 16) {
        fk[(k + 1) & 1] = op.row(tk, 32 * kb, k + 1);
        if (ROT) fl[(k + 1) & 1] = op.row(tk2, 32 * kb, k + 1);
      }
      if (ROT) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fl[k & 1], qf[k], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[k & 1], ql[k], s, 0, 0, 0);
      }
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[k & 1], qf[k], s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    fv[0] = op.row(tv, 32 * kb, 0);
#pragma unroll
    for (int i = 0; i < 16; ++i) dp[i] = nd;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if (k + 1 < D / 16) fv[(k + 1) & 1] = op.row(tv, 32 * kb, k + 1);
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[k & 1], df[k], dp, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    fk[0] = op.column(tk, 32 * kb, 0);
    if (ROT) fl[0] = op.column(tk2, 32 * kb, 0);
    __builtin_amdgcn_sched_barrier(0);
    const int first = 32 * kb + 4 * h2;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float y = ALIBI ? biased(slope, b0 - qpos + first + 8 * (i >> 2) + (i & 3), nl) : nl;
      dp[i] *= fast_exp2(fmaf(s[i], scale_log2, y));
    }
    if (masked) {
      const int last = (causal ? min(nvalid - 1, qpos - b0) : nvalid - 1) - first;
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] = 8 * (i >> 2) + (i & 3) <= last ? dp[i] : 0.f;
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float y[8];
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = dp[8 * k + e];
      split8(y, hi, lo);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int at = k * (D / 32) + db, ahead = at + 1;
        if (ahead < 2 * (D / 32)) {
          fk[ahead & 1] = op.column(tk, 32 * kb + 16 * (ahead / (D / 32)), ahead % (D / 32));
          if (ROT) fl[ahead & 1] = op.column(tk2, 32 * kb + 16 * (ahead / (D / 32)), ahead % (D / 32));
        }
        if (ROT) dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fl[at & 1], as_bf16x8(hi), dq[db], 0, 0, 0);
        dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[at & 1], as_bf16x8(lo), dq[db], 0, 0, 0);
        dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[at & 1], as_bf16x8(hi), dq[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  }
}

// Query gradient of 32 NW packed rows over the 64-key tiles of one key split: NW waves of 32 rows, Q (both parts) and
// dO in registers; K (rotated, both parts) and V pass through LDS, K read by rows and transposed.  Eight waves share a
// tile's loads and rotation where requests fill 256 rows.  Bound like grad_kv, and by the loader's rotation: the same
// ragged requests 2.1 ms for seven products (820 TFLOP/s), the 64-row questions 159 us.  A request in one key split has
// its whole sums here: they are turned back and written at once.
template <int D, int KMI, int NW, int NBUF>
__device__ __forceinline__ void query_gradients(const GradArgs& a, int id, GradQSmem<D, KMI, NBUF>& sm) {
  constexpr int KM = keys_of(KMI), NT = NW * 64;
  constexpr bool ALIBI = KM == kKeysAlibi, ROT = !ALIBI, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  using S = TileLayout<D>;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), h2 = lane >> 5, g = id % a.hkv;
  const GradRowItem item = a.row_items[id / a.hkv];
  const int r = item.request;
  const int qs = a.q_start[r], nrows = (a.q_start[r + 1] - qs) * a.group, shift = a.q_pos0[r] - qs;
  const int pr = item.row0 + 32 * wave + (lane & 31);
  const int src = qs * a.group + min(pr, nrows - 1), tok = token_of(src, a.group_magic), qpos = tok + shift;
  const uint16_t* qrow = a.ws_q + ((int64_t)g * a.rows + src) * D;
  const uint16_t* drow = a.ws_do + ((int64_t)g * a.rows + src) * D;
  const int64_t second = a.hkv * a.rows * D;
  bf16x8 qf[D / 16], ql[D / 16], df[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    qf[s] = as_bf16x8(*reinterpret_cast<const u32x4*>(qrow + 16 * s + 8 * h2));
    if (ROT) ql[s] = as_bf16x8(*reinterpret_cast<const u32x4*>(qrow + second + 16 * s + 8 * h2));
    df[s] = as_bf16x8(*reinterpret_cast<const u32x4*>(drow + 16 * s + 8 * h2));
  }
  const float* in = a.ws_info + (int64_t)g * a.rows + src;
  const float nl = pr < nrows ? in[0] : -INFINITY, nd = in[a.hkv * a.rows];
  const float slope = ALIBI ? natural_slope(a, g * a.group + src - tok * a.group) : 0.f;
  f32x16 dq[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) dq[db] = f32x16{};
  const int qmin = uniform(token_of(qs * a.group + item.row0, a.group_magic) + shift);
  const int qmax = uniform(token_of(qs * a.group + min(item.row0 + 32 * NW, nrows) - 1, a.group_magic) + shift);

  if (ROT) {
    const double rev = revolutions(a, tid % (D / 2));
    if (tid < D / 2) sm.freq[tid] = rev;
    for (int e = tid; e < kAngleRows * (D / 2); e += NT)
      *reinterpret_cast<float2*>(sm.csd + e / (D / 2) * S::CSD_LD + cs_idx<D>(e % (D / 2))) = rope_cs(e / (D / 2), rev);
  }
  __syncthreads();
  TileLoader<D, KMI, NT> ld;
  ld.init(tid);
  TileIter<kSub> it;
  it.init(a.chunks, a.chunk_start[r], a.chunk_start[r + 1], item.split, item.splits);
  bool have = it.seek(a.causal, qmax);
  const auto fetch = [&](const TileIter<kSub>& t) {
    ld.fetch(k_ptr(a.k_pool, t.cur, g, t.j0, D), v_ptr(a.v_pool, t.cur, g, t.j0, D), min(kSub, t.cur.len - t.j0));
  };
  const auto base = [&](float* to, const TileIter<kSub>& t) {
    if (ROT) prefill_base<D, LOCAL>(to, sm.freq, tid, t.cur.pos + (LOCAL ? 0 : t.j0));
  };
  if (have) fetch(it);
  // Eight waves: as in the prefill kernel the upper four store the next tile at the start of a tile's products and the
  // lower four at the end, so that the two waves of a SIMD are in different phases.
  const bool early = NBUF == 2 && NW == 8 && wave >= NW / 2;
  TileIter<kSub> ahead = it;
  bool have_ahead = false;
  if (have && NBUF == 2) {
    base(sm.csb[0][0], it);
    ahead.step();
    have_ahead = ahead.seek(a.causal, qmax);
    if (have_ahead) base(sm.csb[1][0], ahead);
    __syncthreads();
    ld.store(sm.k[0], sm.k[0] + kSub * D, sm.v[0], sm.csb[0][0], sm.csd);
    if (early && have_ahead) fetch(ahead);
    __syncthreads();
  }
  int parity = 0;
  while (have) {
    const int nvalid = min(kSub, it.cur.len - it.j0), b0 = it.cur.pos + it.j0;
    int buf = 0;
    bool have_next;
    if (NBUF == 1) {
      base(sm.csb[0][0], it);
      it.step();
      have_next = it.seek(a.causal, qmax);
      __syncthreads();
      ld.store(sm.k[0], sm.k[0] + kSub * D, sm.v[0], sm.csb[0][0], sm.csd);
      __syncthreads();
      if (have_next) fetch(it);
    } else {
      buf = parity;
      it = ahead;
      have_next = have_ahead;
      if (early && have_next)
        ld.store(sm.k[parity ^ 1], sm.k[parity ^ 1] + kSub * D, sm.v[parity ^ 1], sm.csb[parity ^ 1][0], sm.csd);
      if (have_next) {
        if (!early) fetch(it);
        ahead.step();
        have_ahead = ahead.seek(a.causal, qmax);
        if (early && have_ahead) fetch(ahead);
      }
    }
    grad_tile<D, ALIBI>(sm.k[buf], sm.v[buf], lane, qf, ql, df, dq, a.scale_log2, nl, nd, slope, qpos, b0, nvalid, qmin,
                        a.causal);
    if (NBUF == 2) {
      if (have_ahead) base(sm.csb[parity][0], ahead);
      if (!early && have_next)
        ld.store(sm.k[parity ^ 1], sm.k[parity ^ 1] + kSub * D, sm.v[parity ^ 1], sm.csb[parity ^ 1][0], sm.csd);
      __syncthreads();
      parity ^= 1;
    }
    have = have_next;
  }
  if (item.splits == 1) {  // whole sums: turned back, scaled, rounded and written here, in whole rows through LDS
    __syncthreads();
    constexpr int C = D / 8;
    static_assert(sizeof(sm.k) + sizeof(sm.v) >= NW * 32 * D * sizeof(uint16_t));
    uint16_t* const stage = &sm.k[0][0] + wave * 32 * D;
    const float scale = a.scale_log2 * kLn2;
    const int first = qs * a.group + min(item.row0 + 32 * wave, nrows - 1);
    const int tok0 = uniform(token_of(first, a.group_magic));
    if (ROT && a.rotate_q) {
      float2* const turn = reinterpret_cast<float2*>(stage);
      if (lane < D / 2) turn[lane] = rope_cs(-(tok0 + shift), sm.freq[lane]);
      wait_reads();
      const float* const place = sm.csd + (tok - tok0) * S::CSD_LD;  // 32 rows have at most 32 tokens
#pragma unroll
      for (int db = 0; db < D / 64; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int pair = 32 * db + 8 * (i >> 2) + 4 * h2 + (i & 3);
          float2 cs = *reinterpret_cast<const float2*>(place + cs_idx<D>(pair));
          cs.y = -cs.y;
          float y1, y2;
          rotate_pair(dq[db][i], dq[db + D / 64][i], turn[pair], cs, y1, y2);
          dq[db][i] = y1;
          dq[db + D / 64][i] = y2;
        }
      wait_reads();
    }
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int col = 32 * db + 8 * q4 + 4 * h2;
        const auto at = [&](int d, int e) { return dq[d][4 * q4 + e] * scale; };
        if (!IL)
          *reinterpret_cast<u32x2*>(stage + tile_at<D>(lane & 31, col / 8) + col % 8) =
              u32x2{pack2(at(db, 0), at(db, 1)), pack2(at(db, 2), at(db, 3))};
        else if (db < D / 64)
          *reinterpret_cast<u32x4*>(stage + tile_at<D>(lane & 31, col / 4)) =
              u32x4{pack2(at(db, 0), at(db + D / 64, 0)), pack2(at(db, 1), at(db + D / 64, 1)),
                    pack2(at(db, 2), at(db + D / 64, 2)), pack2(at(db, 3), at(db + D / 64, 3))};
      }
    wait_reads();
#pragma unroll
    for (int i = 0; i < 32 * C / 64; ++i) {
      const int row = (64 * i + lane) / C, chunk = (64 * i + lane) % C, at = item.row0 + 32 * wave + row;
      if (at < nrows) {
        const int to = qs * a.group + at, token = token_of(to, a.group_magic);
        *reinterpret_cast<u32x4*>(a.dq + ((int64_t)token * a.hq + g * a.group + to - token * a.group) * D + 8 * chunk) =
            *reinterpret_cast<const u32x4*>(stage + tile_at<D>(row, chunk));
      }
    }
    return;
  }
  if (pr >= nrows) return;
  float* out = a.ws_dq + (((int64_t)item.split * a.hkv + g) * a.rows + src) * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      *reinterpret_cast<f32x4*>(out + 32 * db + 8 * q4 + 4 * h2) =
          f32x4{dq[db][4 * q4], dq[db][4 * q4 + 1], dq[db][4 * q4 + 2], dq[db][4 * q4 + 3]};
}
template <int D, int KMI, int NW, int NBUF>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void grad_q(GradArgs a) {
  __shared__ GradQSmem<D, KMI, NBUF> sm;
  query_gradients<D, KMI, NW, NBUF>(a, blockIdx.x, sm);
}
// Both in one launch, the first `tiles` workgroups for keys and values.
template <int D, int KMI>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void grad_all(GradArgs a, int tiles) {
  __shared__ union {
    KeySmem<D, KMI> keys;
    GradQSmem<D, KMI, 1> queries;
  } sm;
  if ((int)blockIdx.x < tiles)
    key_gradients<D, KMI>(a, blockIdx.x, sm.keys);
  else
    query_gradients<D, KMI, 4, 1>(a, blockIdx.x - tiles, sm.queries);
}

// Keys of a tile's parts that a workgroup sums, and workgroups a (tile, KV head).
constexpr int kMergeRows = 32, kMergeBlocks = 2 * kGradHalves * kGradTileKeys / kMergeRows;

// Partial results added up in their order, two kinds of workgroups in one launch.  The first `blocks`: partial query
// gradients of a block of tokens, turned back from the rows' positions, scaled, rounded.  The others: 32 rows of the
// key or value gradients of a tile whose uses were cut into parts.  D / 16 threads a row.  Bound by memory (12 us for
// 512 tokens of 32 heads of 128 in four splits, 38 MB).
template <int D, bool IL>
__global__ __launch_bounds__(256) void finish(GradArgs a, int blocks) {
  constexpr int TPR = D / 16;
  const int t0 = 8 * (threadIdx.x % TPR);
  const auto sum = [&](const float* p, int64_t stride, int count, float (&lo)[8], float (&hi)[8]) {
    for (int s0 = 0; s0 < count; s0 += 4) {
      f32x4 x[4][4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const float* src = p + min(s0 + s, count - 1) * stride + t0;
        x[s][0] = reinterpret_cast<const f32x4*>(src)[0];
        x[s][1] = reinterpret_cast<const f32x4*>(src)[1];
        x[s][2] = reinterpret_cast<const f32x4*>(src + D / 2)[0];
        x[s][3] = reinterpret_cast<const f32x4*>(src + D / 2)[1];
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (s0 + s >= count) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          lo[e] += x[s][e >> 2][e & 3];
          hi[e] += x[s][2 + (e >> 2)][e & 3];
        }
      }
    }
  };
  if ((int)blockIdx.x >= blocks) {
    const int id = blockIdx.x - blocks, g = id / kMergeBlocks % a.hkv;
    const GradMerge* const m = a.merges + id / (kMergeBlocks * a.hkv);
    for (int i = threadIdx.x / TPR; i < kMergeRows; i += 256 / TPR) {
      const int row = id % kMergeBlocks * kMergeRows + i, key = row % kGradTileKeys;
      const GradHalf h = m->half[row / (2 * kGradTileKeys)];
      if (key >= h.keys) continue;
      float lo[8] = {}, hi[8] = {};
      const int64_t stride = (int64_t)a.hkv * 2 * kGradHalves * kGradTileKeys * D;
      sum(a.ws_parts + m->part * stride + ((int64_t)g * 2 * kGradHalves * kGradTileKeys + row) * D, stride, m->parts, lo,
          hi);
      if (row / kGradTileKeys % 2)
        store_pairs<D, false>(a.dv_pool + h.v_off + ((int64_t)g * h.vst + key) * D, t0, lo, hi);
      else
        store_pairs<D, IL>(a.dk_pool + h.k_off + ((int64_t)g * h.kst + key) * D, t0, lo, hi);
    }
    return;
  }
  __shared__ float2 cs[kMaxBlockTokens][D / 2];
  const GradBlock b = a.blocks[blockIdx.x];
  if (b.splits == 1) return;  // written with its sums
  if (a.rotate_q) {
    for (int e = threadIdx.x; e < b.tokens * (D / 2); e += 256)
      cs[e / (D / 2)][e % (D / 2)] = rope_cs(-(b.t0 + e / (D / 2) + b.pos_shift), revolutions(a, e % (D / 2)));
    __syncthreads();
  }
  for (int row = threadIdx.x / TPR; row < b.tokens * a.hq; row += 256 / TPR) {
    const int tok = row / a.hq, h = row % a.hq;
    const int64_t src = (int64_t)(h / a.group) * a.rows + (int64_t)(b.t0 + tok) * a.group + h % a.group;
    float lo[8] = {}, hi[8] = {};
    sum(a.ws_dq + src * D, a.hkv * a.rows * D, b.splits, lo, hi);
    const float scale = a.scale_log2 * kLn2;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] *= scale;
      hi[e] *= scale;
      if (a.rotate_q) rotate_by(lo[e], hi[e], cs[tok][t0 + e], lo[e], hi[e]);
    }
    store_pairs<D, IL>(a.dq + ((int64_t)(b.t0 + tok) * a.hq + h) * D, t0, lo, hi);
  }
}

template <int D, int KMI>
hipError_t launch(const GradArgs& a, const lazy_backward_info_t& i, hipStream_t stream) {
  constexpr bool IL = interleaved_of(KMI);
  if (i.num_blocks) prepare_rows<D, IL><<<i.num_blocks, 256, 0, stream>>>(a);
  const int tiles = i.num_tiles * a.hkv, items = i.num_row_items * a.hkv;
  if (i.row_blocks == 1) {
    if (tiles + items) grad_all<D, KMI><<<tiles + items, 256, 0, stream>>>(a, tiles);
  } else if constexpr (D == 128) {
    if (tiles) grad_kv<D, KMI><<<tiles, 256, 0, stream>>>(a);
    if (items) grad_q<D, KMI, 8, 2><<<items, 512, 0, stream>>>(a);
  }
  const int merges = i.num_merges * a.hkv * kMergeBlocks, blocks = i.row_slots > 1 ? i.num_blocks : 0;
  if (blocks + merges) finish<D, IL><<<blocks + merges, 256, 0, stream>>>(a, blocks);
  return hipGetLastError();
}

template <int D>
hipError_t launch_mode(const GradArgs& a, int keys, bool interleaved, const lazy_backward_info_t& i, hipStream_t s) {
  if (keys == kKeysAlibi) return launch<D, kKeysAlibi>(a, i, s);
  if (keys == kKeysLocal)
    return interleaved ? launch<D, kKeysLocal | kInterleaved>(a, i, s) : launch<D, kKeysLocal>(a, i, s);
  return interleaved ? launch<D, kKeysNope | kInterleaved>(a, i, s) : launch<D, kKeysNope>(a, i, s);
}

}  // namespace

hipError_t launch_backward(const GradArgs& a, int head_dim, bool local_keys, bool interleaved, bool alibi,
                           const lazy_backward_info_t& info, hipStream_t stream) {
  const int keys = alibi ? kKeysAlibi : local_keys ? kKeysLocal : kKeysNope;
  return head_dim == 64 ? launch_mode<64>(a, keys, interleaved, info, stream)
                        : launch_mode<128>(a, keys, interleaved, info, stream);
}

}  // namespace lazy
