// Backward pass of the prefill attention for gfx950: gradients of the queries and of the stored keys and values.
//
// Four launches.  (1) prepare_rows: queries rotated to their positions, times scale * log2 e, in bf16 and packed by KV
// head (row = token * G + head in group), and two numbers a row, -lse log2 e and -delta.  (2) grad_kv: dk and dv, one
// 64-key tile of the store at a time.  (3) grad_q: partial dq, one row tile and key split at a time.  (4) finish_rows:
// partial dq summed, turned back and rounded (and merge_tiles: the same for tiles whose uses were cut into parts).
// The probabilities are recomputed in (2) and in (3): seven products of the two kernels against five if dq were summed
// over key tiles with atomics, whose order would change results from call to call.
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

// Queries rotated, scaled and packed by KV head; row constants.  One workgroup a block of tokens, D / 16 threads a row.
template <int D, bool IL>
__global__ __launch_bounds__(256) void prepare_rows(GradArgs a) {
  __shared__ float2 cs[kMaxBlockTokens][D / 2];
  const GradBlock b = a.blocks[blockIdx.x];
  if (a.rotate_q) {
    for (int e = threadIdx.x; e < b.tokens * (D / 2); e += 256) {
      const int t = e % (D / 2);
      cs[e / (D / 2)][t] = rope_cs(b.t0 + e / (D / 2) + b.pos_shift, theta_rev(t, D, a.rope_log2_base, a.inv_freq));
    }
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
    float yl[8], yh[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      yl[e] = element(lo, e);
      yh[e] = element(hi, e);
      if (a.rotate_q) rotate_by(element(lo, e), element(hi, e), cs[tok][t0 + e], yl[e], yh[e]);
      yl[e] *= a.scale_log2;
      yh[e] *= a.scale_log2;
    }
    store_pairs<D, false>(a.ws_q + dst * D, t0, yl, yh);
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(a.dout + src * D + 2 * t0 + 8 * k);
      const u32x4 y = *reinterpret_cast<const u32x4*>(a.out + src * D + 2 * t0 + 8 * k);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(element(x, e), element(y, e), sum);
    }
#pragma unroll
    for (int m = 1; m < TPR; m <<= 1) sum += __shfl_xor(sum, m, 64);
    if (t0 == 0) {
      const float lse = a.lse[src];
      if (a.dlse) sum -= a.dlse[src];
      // A row that sees no key: exp2(score - inf) = 0.
      a.ws_info[dst] = make_float2(lse == -INFINITY ? -INFINITY : -lse * 1.4426950408889634f, -sum);
    }
  }
}

// Key and value gradients.  A workgroup is one wave and owns the 64 keys of a tile: K (rotated) and V stay in registers
// as the right-hand operands of S = Q K^T and dP = dO V^T, whose accumulators have a key in every lane and 32 query
// rows in registers and lane halves; P and dS leave them as the right-hand operands of dV^T += dO^T P and
// dK^T += Q^T dS without any exchange between lanes.  Q and dO come through LDS, 32 rows at a time, read by rows for
// the first two products and transposed for the last two.  -lse and -delta are the accumulators' initial values.
// dK is kept in the rotated frame of the use at hand and turned on when the next use has another position.
template <int D, int KMI>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(1, 1))) void grad_kv(GradArgs a) {
  constexpr int KM = keys_of(KMI);
  constexpr bool ALIBI = KM == kKeysAlibi, ROT = !ALIBI, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  constexpr int C = D / 8;
  __shared__ uint16_t tq[kGradRows * D] __attribute__((aligned(16)));
  __shared__ uint16_t td[kGradRows * D] __attribute__((aligned(16)));
  __shared__ float nlse[kGradRows] __attribute__((aligned(16)));
  __shared__ float ndelta[kGradRows] __attribute__((aligned(16)));
  __shared__ int rpos[kGradRows] __attribute__((aligned(16)));
  __shared__ float rslope[kGradRows] __attribute__((aligned(16)));
  __shared__ double freq[D / 2];
  __shared__ float2 turn[D / 2] __attribute__((aligned(16)));
  const int lane = threadIdx.x, h2 = lane >> 5, g = blockIdx.x % a.hkv;
  const GradTile t = a.tiles[blockIdx.x / a.hkv];
  if (ROT && lane < D / 2) freq[lane] = theta_rev(lane, D, a.rope_log2_base, a.inv_freq);
  __syncthreads();

  bf16x8 kf[2][D / 16], vf[2][D / 16];
  f32x16 dk[2][D / 32], dv[2][D / 32];
  int key[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    key[b] = 32 * b + (lane & 31);
    const uint16_t* v = a.v_pool + t.v_off + ((int64_t)g * t.vst + min(key[b], t.keys - 1)) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) vf[b][s] = as_bf16x8(*reinterpret_cast<const u32x4*>(v + 16 * s + 8 * h2));
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[b][db] = dv[b][db] = f32x16{};
  }
  const uint16_t* qbase = a.ws_q + (int64_t)g * a.rows * D;
  const float2* ibase = a.ws_info + (int64_t)g * a.rows;
  const int head0 = g * a.group;
  int frame = 0;  // position by which dk is rotated (NoPE: that of the tile's key 0)
  for (int si = t.seg_begin; si < t.seg_end; ++si) {
    const GradSeg seg = a.segs[si];
    const int here = LOCAL ? seg.record_pos : seg.pos;
#pragma unroll
    for (int b = 0; b < 2; ++b)
      load_keys<D, KM, IL>(a.k_pool + t.k_off + ((int64_t)g * t.kst + min(key[b], t.keys - 1)) * D, h2,
                           LOCAL ? here : here + key[b], freq, kf[b]);
    if (ROT && si > t.seg_begin && here != frame) {
      __syncthreads();
      if (lane < D / 2) turn[lane] = rope_cs(here - frame, freq[lane]);
      __syncthreads();
#pragma unroll
      for (int db = 0; db < D / 64; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float2 cs = turn[32 * db + 8 * (i >> 2) + 4 * h2 + (i & 3)];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const float x1 = dk[b][db][i], x2 = dk[b][db + D / 64][i];
            float y1, y2;
            rotate_by(x1, x2, cs, y1, y2);
            dk[b][db][i] = y1;
            dk[b][db + D / 64][i] = y2;
          }
        }
    }
    frame = here;

    for (int row0 = seg.row_begin; row0 < seg.row_end; row0 += kGradRows) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kGradRows * C / 64; ++i) {
        const int e = 64 * i + lane, row = e / C, chunk = e % C;
        const int src = min(row0 + row, seg.row_end - 1);
        const int tok = token_of(src, a.group_magic);
        *reinterpret_cast<u32x4*>(tq + tile_at<D>(row, chunk)) =
            *reinterpret_cast<const u32x4*>(qbase + (int64_t)src * D + 8 * chunk);
        *reinterpret_cast<u32x4*>(td + tile_at<D>(row, chunk)) = *reinterpret_cast<const u32x4*>(
            a.dout + ((int64_t)tok * (a.hq - a.group) + src + head0) * D + 8 * chunk);
      }
      if (lane < kGradRows) {
        const int src = row0 + lane;
        const int tok = token_of(src, a.group_magic);
        const float2 in = src < seg.row_end ? ibase[src] : make_float2(-INFINITY, 0.f);
        nlse[lane] = in.x;
        ndelta[lane] = in.y;
        rpos[lane] = tok + seg.pos_shift;
        if (ALIBI) rslope[lane] = alibi_slope(head0 + src - tok * a.group, a.hq, a.inv_freq, 1.f);
      }
      __syncthreads();

      f32x16 s[2], dp[2];
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(nlse + 8 * q4 + 4 * h2);
        const f32x4 y = *reinterpret_cast<const f32x4*>(ndelta + 8 * q4 + 4 * h2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[0][4 * q4 + e] = s[1][4 * q4 + e] = x[e];
          dp[0][4 * q4 + e] = dp[1][4 * q4 + e] = y[e];
        }
      }
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const bf16x8 fq = row_operand<D>(tq, lane & 31, k, h2), fd = row_operand<D>(td, lane & 31, k, h2);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq, kf[b][k], s[b], 0, 0, 0);
          dp[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd, vf[b][k], dp[b], 0, 0, 0);
        }
      }
      const bool masked = row0 < seg.full_from;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (ALIBI) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = 8 * (i >> 2) + 4 * h2 + (i & 3);
            s[b][i] = fmaf(rslope[row], (float)(seg.pos + key[b] - rpos[row]), s[b][i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = fast_exp2(s[b][i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) dp[b][i] *= s[b][i];
        if (masked) {
          const bool used = key[b] >= seg.key_begin && key[b] < seg.key_end;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = 8 * (i >> 2) + 4 * h2 + (i & 3);
            const bool ok = used && (!a.causal || seg.pos + key[b] <= rpos[row]);
            s[b][i] = ok ? s[b][i] : 0.f;
            dp[b][i] = ok ? dp[b][i] : 0.f;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 pf[2], sf[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float x[8], y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = s[b][8 * k + e];
            y[e] = dp[b][8 * k + e];
          }
          pf[b] = as_bf16x8(pack8(x));
          sf[b] = as_bf16x8(pack8(y));
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const bf16x8 fd = column_operand<D>(td, 16 * k, db, lane), fq = column_operand<D>(tq, 16 * k, db, lane);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            dv[b][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd, pf[b], dv[b][db], 0, 0, 0);
            dk[b][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq, sf[b], dk[b][db], 0, 0, 0);
          }
        }
      }
    }
  }

  // q carries scale * log2 e, dk wants scale: a factor of ln 2.  Turned back to the frame in which the key is stored.
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int db = 0; db < D / 64; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x1 = dk[b][db][i] * kLn2, x2 = dk[b][db + D / 64][i] * kLn2;
        if (ROT) {
          const int pair = 32 * db + 8 * (i >> 2) + 4 * h2 + (i & 3);
          rotate_by(x1, x2, rope_cs(-(LOCAL ? frame : frame + key[b]), freq[pair]), x1, x2);
        }
        dk[b][db][i] = x1;
        dk[b][db + D / 64][i] = x2;
      }
    if (t.part >= 0) {
      float* out = a.ws_parts + (((int64_t)t.part * a.hkv + g) * 2 * kGradTileKeys + key[b]) * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int col = 32 * db + 8 * q4 + 4 * h2;
          *reinterpret_cast<f32x4*>(out + col) =
              f32x4{dk[b][db][4 * q4], dk[b][db][4 * q4 + 1], dk[b][db][4 * q4 + 2], dk[b][db][4 * q4 + 3]};
          *reinterpret_cast<f32x4*>(out + kGradTileKeys * D + col) =
              f32x4{dv[b][db][4 * q4], dv[b][db][4 * q4 + 1], dv[b][db][4 * q4 + 2], dv[b][db][4 * q4 + 3]};
        }
    } else if (key[b] < t.keys) {
      uint16_t* ko = a.dk_pool + t.k_off + ((int64_t)g * t.kst + key[b]) * D;
      uint16_t* vo = a.dv_pool + t.v_off + ((int64_t)g * t.vst + key[b]) * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int col = 32 * db + 8 * q4 + 4 * h2;
          *reinterpret_cast<u32x2*>(vo + col) = u32x2{pack2(dv[b][db][4 * q4], dv[b][db][4 * q4 + 1]),
                                                      pack2(dv[b][db][4 * q4 + 2], dv[b][db][4 * q4 + 3])};
          if (!IL) {
            *reinterpret_cast<u32x2*>(ko + col) = u32x2{pack2(dk[b][db][4 * q4], dk[b][db][4 * q4 + 1]),
                                                        pack2(dk[b][db][4 * q4 + 2], dk[b][db][4 * q4 + 3])};
          } else if (db < D / 64) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2(dk[b][db][4 * q4 + e], dk[b][db + D / 64][4 * q4 + e]);
            *reinterpret_cast<u32x4*>(ko + 2 * col) = w;
          }
        }
    }
  }
}

// Sum of a tile's parts, in their order.  Workgroup: one (tile, KV head); D / 16 threads a key.
template <int D, bool IL>
__global__ __launch_bounds__(256) void merge_tiles(GradArgs a) {
  const int g = blockIdx.x % a.hkv;
  const GradMerge m = a.merges[blockIdx.x / a.hkv];
  constexpr int TPR = D / 16;
  const int t0 = 8 * (threadIdx.x % TPR);
  for (int row = threadIdx.x / TPR; row < 2 * kGradTileKeys; row += 256 / TPR) {
    const bool values = row >= kGradTileKeys;
    const int key = row % kGradTileKeys;
    if (key >= m.keys) continue;
    float lo[8] = {}, hi[8] = {};
    for (int p = m.part; p < m.part + m.parts; ++p) {
      const float* src = a.ws_parts + (((int64_t)p * a.hkv + g) * 2 * kGradTileKeys + row) * D + t0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] += src[e];
        hi[e] += src[D / 2 + e];
      }
    }
    if (values)
      store_pairs<D, false>(a.dv_pool + m.v_off + ((int64_t)g * m.vst + key) * D, t0, lo, hi);
    else
      store_pairs<D, IL>(a.dk_pool + m.k_off + ((int64_t)g * m.kst + key) * D, t0, lo, hi);
  }
}

// Query gradient of 128 RB packed rows over the 64-key tiles of one key split: four waves of RB blocks of 32 rows, Q
// and dO in registers.  S^T = K Q^T and dP^T = V dO^T have a query row in every lane; dS^T leaves them as the right-hand
// operand of dQ^T += K^T dS^T.  K (rotated) and V pass through LDS, K read by rows and transposed.
template <int D, int KMI, int RB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 2))) void grad_q(GradArgs a) {
  constexpr int KM = keys_of(KMI);
  constexpr bool ALIBI = KM == kKeysAlibi, ROT = !ALIBI, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  constexpr int PP = D / 8;  // pairs of a key row that one of its four loader threads rotates
  __shared__ uint16_t tk[kSub * D] __attribute__((aligned(16)));
  __shared__ uint16_t tv[kSub * D] __attribute__((aligned(16)));
  __shared__ double freq[D / 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h2 = lane >> 5, g = blockIdx.x % a.hkv;
  const GradRowItem item = a.row_items[blockIdx.x / a.hkv];
  const int r = item.request;
  const int qs = a.q_start[r], nrows = (a.q_start[r + 1] - qs) * a.group, shift = a.q_pos0[r] - qs;
  if (ROT && tid < D / 2) freq[tid] = theta_rev(tid, D, a.rope_log2_base, a.inv_freq);

  bf16x8 qf[RB][D / 16], df[RB][D / 16];
  float nl[RB], nd[RB], slope[RB];
  int row[RB], qpos[RB];
  f32x16 dq[RB][D / 32];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int pr = item.row0 + 32 * (RB * wave + rb) + (lane & 31);
    row[rb] = pr < nrows ? qs * a.group + pr : -1;
    const int src = qs * a.group + min(pr, nrows - 1);
    const int tok = token_of(src, a.group_magic);
    qpos[rb] = tok + shift;
    const uint16_t* qrow = a.ws_q + ((int64_t)g * a.rows + src) * D;
    const uint16_t* drow = a.dout + ((int64_t)tok * (a.hq - a.group) + src + g * a.group) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      qf[rb][s] = as_bf16x8(*reinterpret_cast<const u32x4*>(qrow + 16 * s + 8 * h2));
      df[rb][s] = as_bf16x8(*reinterpret_cast<const u32x4*>(drow + 16 * s + 8 * h2));
    }
    const float2 in = a.ws_info[(int64_t)g * a.rows + src];
    nl[rb] = pr < nrows ? in.x : -INFINITY;
    nd[rb] = in.y;
    slope[rb] = ALIBI ? alibi_slope(g * a.group + src - tok * a.group, a.hq, a.inv_freq, 1.f) : 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dq[rb][db] = f32x16{};
  }
  const int first_tok = token_of(item.row0, a.group_magic);
  const int last_tok = token_of(min(item.row0 + 128 * RB, nrows) - 1, a.group_magic);
  const int qmin = uniform(qs + first_tok + shift), qmax = uniform(qs + last_tok + shift);

  TileIter<kSub> it;
  it.init(a.chunks, a.chunk_start[r], a.chunk_start[r + 1], item.split, item.splits);
  const int krow = tid >> 2, part = tid & 3;
  while (it.seek(a.causal, qmax)) {
    const int nvalid = min(kSub, it.cur.len - it.j0), b0 = it.cur.pos + it.j0;
    __syncthreads();
    {
      const int kr = min(krow, nvalid - 1);
      const uint16_t* ks = k_ptr(a.k_pool, it.cur, g, it.j0 + kr, D);
      const uint16_t* vs = v_ptr(a.v_pool, it.cur, g, it.j0 + kr, D);
#pragma unroll
      for (int v = 0; v < PP / 8; ++v) {
        const int t0 = part * PP + 8 * v;
        u32x4 lo, hi;
        load_pairs<D, IL>(ks, t0, lo, hi);
        if (ROT) {
          float yl[8], yh[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            rotate_by(element(lo, e), element(hi, e), rope_cs(LOCAL ? it.cur.pos : b0 + krow, freq[t0 + e]), yl[e],
                      yh[e]);
          lo = pack8(yl);
          hi = pack8(yh);
        }
        *reinterpret_cast<u32x4*>(tk + tile_at<D>(krow, t0 / 8)) = lo;
        *reinterpret_cast<u32x4*>(tk + tile_at<D>(krow, D / 16 + t0 / 8)) = hi;
      }
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        *reinterpret_cast<u32x4*>(tv + tile_at<D>(krow, part * (D / 32) + i)) =
            *reinterpret_cast<const u32x4*>(vs + 8 * (part * (D / 32) + i));
    }
    __syncthreads();
    const bool masked = nvalid < kSub || (a.causal && b0 + kSub - 1 > qmin);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s[RB], dp[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[rb][i] = nl[rb];
          dp[rb][i] = nd[rb];
        }
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const bf16x8 fk = row_operand<D>(tk, 32 * kb + (lane & 31), k, h2);
        const bf16x8 fv = row_operand<D>(tv, 32 * kb + (lane & 31), k, h2);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk, qf[rb][k], s[rb], 0, 0, 0);
          dp[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv, df[rb][k], dp[rb], 0, 0, 0);
        }
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int kk = 32 * kb + 8 * (i >> 2) + 4 * h2 + (i & 3);
          if (ALIBI) s[rb][i] = fmaf(slope[rb], (float)(b0 + kk - qpos[rb]), s[rb][i]);
          dp[rb][i] *= fast_exp2(s[rb][i]);
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int kk = 32 * kb + 8 * (i >> 2) + 4 * h2 + (i & 3);
            const bool ok = kk < nvalid && (!a.causal || b0 + kk <= qpos[rb]);
            dp[rb][i] = ok ? dp[rb][i] : 0.f;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 sf[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = dp[rb][8 * k + e];
          sf[rb] = as_bf16x8(pack8(y));
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const bf16x8 fk = column_operand<D>(tk, 32 * kb + 16 * k, db, lane);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            dq[rb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk, sf[rb], dq[rb][db], 0, 0, 0);
        }
      }
    }
    it.step();
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (row[rb] < 0) continue;
    float* out = a.ws_dq + (((int64_t)item.split * a.hkv + g) * a.rows + row[rb]) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<f32x4*>(out + 32 * db + 8 * q4 + 4 * h2) =
            f32x4{dq[rb][db][4 * q4], dq[rb][db][4 * q4 + 1], dq[rb][db][4 * q4 + 2], dq[rb][db][4 * q4 + 3]};
  }
}

// Partial query gradients summed in the order of the splits, turned back from the rows' positions, scaled, rounded.
template <int D, bool IL>
__global__ __launch_bounds__(256) void finish_rows(GradArgs a) {
  __shared__ float2 cs[kMaxBlockTokens][D / 2];
  const GradBlock b = a.blocks[blockIdx.x];
  if (a.rotate_q) {
    for (int e = threadIdx.x; e < b.tokens * (D / 2); e += 256) {
      const int t = e % (D / 2);
      cs[e / (D / 2)][t] = rope_cs(-(b.t0 + e / (D / 2) + b.pos_shift), theta_rev(t, D, a.rope_log2_base, a.inv_freq));
    }
    __syncthreads();
  }
  constexpr int TPR = D / 16;
  const int t0 = 8 * (threadIdx.x % TPR);
  for (int row = threadIdx.x / TPR; row < b.tokens * a.hq; row += 256 / TPR) {
    const int tok = row / a.hq, h = row % a.hq;
    const int64_t src = (int64_t)(h / a.group) * a.rows + (int64_t)(b.t0 + tok) * a.group + h % a.group;
    float lo[8] = {}, hi[8] = {};
    for (int s = 0; s < b.splits; ++s) {
      const float* p = a.ws_dq + ((int64_t)s * a.hkv * a.rows + src) * D + t0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] += p[e];
        hi[e] += p[D / 2 + e];
      }
    }
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
  if (i.num_tiles) grad_kv<D, KMI><<<i.num_tiles * a.hkv, 64, 0, stream>>>(a);
  if (i.num_merges) merge_tiles<D, IL><<<i.num_merges * a.hkv, 256, 0, stream>>>(a);
  if (i.num_row_items) {
    if (i.row_blocks == 2)
      grad_q<D, KMI, 2><<<i.num_row_items * a.hkv, 256, 0, stream>>>(a);
    else
      grad_q<D, KMI, 1><<<i.num_row_items * a.hkv, 256, 0, stream>>>(a);
    finish_rows<D, IL><<<i.num_blocks, 256, 0, stream>>>(a);
  }
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
