// Eviction by accumulated attention weight for gfx950: key weights of prompts and of single tokens, the selection of the
// heaviest keys, and the gathering of the kept ones.
//
// Key weights are sums that later calls go on with and that ranks are taken of, so their scores are formed more exactly
// than an attention output needs: rotated queries and keys are each kept as two bf16 parts (2^-16 instead of 2^-8), and a
// score is the sum of three products, first x first and the two mixed ones; single tokens with few heads to a key take
// products of 32 bits instead.  With one part each, sums over 8 to 32 heads were 1e-4 to 5e-4 off (2-norm), now 2e-8 to
// 4e-7.  ALiBi rotates nothing: one part is exact.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "lazy_attn_device.h"
#include "lazy_attn_internal.h"
#include "lazy_attn_params.h"
#include "lazy_attn_tiles.h"

namespace lazy {
namespace {

// A request's 64-key tiles with the index of each tile's first key among the request's keys.
struct KeyIter : TileIter<kSub> {
  int base;  // index of the current record's key 0
  __device__ void start(const lazy_chunk_t* table, int c0, int c1, int split, int splits) {
    const First first = first_block(table, c0, c1);
    init(table, c0, c1, split, splits, first);
    const int lane = threadIdx.x & 63;
    int sum = 0;  // keys of the records before i
#pragma unroll
    for (int u = 0; u < 4; ++u) sum += c0 + 64 * u + lane < i ? (u == 0 ? first.mine.len : first.len[u - 1]) : 0;
    for (int k = c0 + 256 + lane; k < i; k += 64) sum += table[k].len;
    base = __builtin_amdgcn_readlane(wave_incl_scan(sum), 63);
  }
  __device__ void next() {
    --left;
    j0 += kSub;
    while (left > 0 && j0 >= cur.len) {
      base += cur.len;
      ++i;
      j0 = 0;
      cur = nxt;
      if (i + 1 < end) nxt = load_rec(recs + i + 1);
    }
  }
  __device__ void skip(int n) {
    for (int k = 0; k < n && left > 0; ++k) next();
  }
};

constexpr int kPrepTokens = 2;

// Queries rotated, in two parts, packed by KV head, and -lse (times log2 e but for ALiBi) of each row; workgroups past the last block (NoPE keys
// only) write the table of angles.
template <int D, int KMI>
__global__ __launch_bounds__(256) void prepare_queries(WeightArgs a, int blocks) {
  constexpr bool IL = interleaved_of(KMI);
  __shared__ float2 cs[kPrepTokens][D / 2];
  if ((int)blockIdx.x >= blocks) {
    angle_rows<D>(a, blockIdx.x - blocks);
    return;
  }
  const int first = blockIdx.x * kPrepTokens, tokens = min(kPrepTokens, a.total_q - first);
  if (a.rotate_q) {
    for (int e = threadIdx.x; e < tokens * (D / 2); e += 256) {
      const int t = e % (D / 2), tok = first + e / (D / 2);
      int lo = 0, hi = a.batch;  // the last request that starts at or before the token (empty ones come before it)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_start[mid] <= tok)
          lo = mid;
        else
          hi = mid;
      }
      cs[e / (D / 2)][t] = rope_cs(a.q_pos0[lo] + tok - a.q_start[lo], revolutions(a, t));
    }
    __syncthreads();
  }
  constexpr int TPR = D / 16;
  const int t0 = 8 * (threadIdx.x % TPR);
  for (int row = threadIdx.x / TPR; row < tokens * a.hq; row += 256 / TPR) {
    const int tok = row / a.hq, h = row % a.hq;
    const int64_t src = (int64_t)(first + tok) * a.hq + h;
    const int64_t dst = (int64_t)(h / a.group) * a.rows + (int64_t)(first + tok) * a.group + h % a.group;
    u32x4 lo, hi;
    load_pairs<D, IL>(a.q + src * D, t0, lo, hi);
    const float lse = a.lse[src];
    if (lse == -INFINITY) lo = hi = u32x4{};  // a row that gives nothing, whatever stands in it: exp2(0 - inf) = 0
    if (a.rotate_k) {
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
      *reinterpret_cast<u32x4*>(second + t0) = rest;
      split8(yh, hi, rest);
      *reinterpret_cast<u32x4*>(second + D / 2 + t0) = rest;
    }
    *reinterpret_cast<u32x4*>(a.ws_q + dst * D + t0) = lo;
    *reinterpret_cast<u32x4*>(a.ws_q + dst * D + D / 2 + t0) = hi;
    if (t0 == 0) a.ws_nlse[dst] = lse == -INFINITY ? -INFINITY : -lse * lse_scale(keys_of(KMI));
  }
}

// Weights of a prompt: workgroup (key split and row split, KV head, request), two 64-key tiles at a time, 32 keys a wave,
// whose rotated parts stay in registers while the rows of the request pass through LDS, 32 at a time, copied to the other
// of two buffers during the products.  S = Q K^T has a key in every lane and 32 rows in registers and lane halves, so a
// key's sum never leaves its lane.  Bound by the three products: 4 requests of 256 rows and 33K keys 750 us, 828 GFLOP at
// 1.10 PFLOP/s (the large library product: 1.22); 8 of 64 rows and 5.3K keys 84 us (0.79), where a tile's loads and
// rotation serve 8 steps only.  Four tiles a workgroup: with 6, 8 or 12 the latter took 92, 84 and 109 us, the former the
// same to 10% more.
constexpr int kStepRows = 32;
template <int D, int KMI>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3))) void weigh_prompt(WeightArgs a) {
  constexpr int KM = keys_of(KMI);
  constexpr bool ALIBI = KM == kKeysAlibi, ROT = !ALIBI, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  constexpr int C = D / 8, COPIES = kStepRows * C / 256, PARTS = ROT ? 2 : 1;
  __shared__ uint16_t tq0[PARTS * kStepRows * D] __attribute__((aligned(16)));
  __shared__ float nl0[kStepRows] __attribute__((aligned(16)));
  __shared__ uint16_t tq1[PARTS * kStepRows * D] __attribute__((aligned(16)));
  __shared__ float nl1[kStepRows] __attribute__((aligned(16)));
  __shared__ int rpos_all[4][kStepRows] __attribute__((aligned(16)));
  __shared__ float rslope_all[4][kStepRows] __attribute__((aligned(16)));
  __shared__ float2 turn_all[4][D / 2] __attribute__((aligned(16)));
  // Angles of positions 0 .. 31, one row each; 16-byte chunk c of row r at place c ^ (r % 16).
  __shared__ float trows[KM == kKeysNope ? 32 * D : 4] __attribute__((aligned(16)));
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), h2 = lane >> 5;
  const int r = blockIdx.z, g = blockIdx.y, split = blockIdx.x % a.splits, rs = blockIdx.x / a.splits;
  const int qs = a.q_start[r], nrows = (a.q_start[r + 1] - qs) * a.group, shift = a.q_pos0[r] - qs;
  const int steps = (nrows + kStepRows - 1) / kStepRows;
  const int row_begin = qs * a.group + (int)((int64_t)steps * rs / a.row_splits) * kStepRows;
  const int row_end = qs * a.group + min(nrows, (int)((int64_t)steps * (rs + 1) / a.row_splits) * kStepRows);
  const int room = min(a.key_start[r + 1], a.num_keys) - a.key_start[r];
  const double rev = ROT ? revolutions(a, lane % (D / 2)) : 0.0;
  const uint16_t* qbase = a.ws_q + (int64_t)g * a.rows * D;
  const int64_t second = a.hkv * a.rows * D;
  const float* nbase = a.ws_nlse + (int64_t)g * a.rows;
  const auto fetch = [&](int row0, uint16_t* tq, float* nl) {
    const int most = row_end - 1 - row0;  // rows past the end repeat the last one; they are masked
    const int e0 = again(tid);
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const int row = (256 * i + e0) / C, chunk = ((256 * i + e0) % C) ^ swizzle<D>(row);
      const uint16_t* src = qbase + (int64_t)row0 * D + min(row, most) * D + 8 * chunk;
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        copy_async(src + part * second, tq + part * kStepRows * D + 2048 * i + 512 * wave);
    }
    if (tid < kStepRows) copy_async4(nbase + row0 + min(e0, most), nl);
  };
  if (KM == kKeysNope) {
    const int e0 = again(tid);
#pragma unroll
    for (int i = 0; i < 32 * D / 1024; ++i) {
      const int row = (256 * i + e0) / (D / 4), chunk = ((256 * i + e0) % (D / 4)) ^ (row & 15);
      copy_async(a.ws_angles + row * D + 4 * chunk, trows + 1024 * i + 256 * wave);
    }
  }
  if (row_begin < row_end) fetch(row_begin, tq0, nl0);
  KeyIter it;
  it.start(a.chunks, a.chunk_start[r], a.chunk_start[r + 1], split, a.splits);
  const int rounds = (it.left + 1) / 2;
  it.skip(wave >> 1);
  __syncthreads();
  float* part = a.ws_part + (int64_t)(rs * a.hkv + g) * a.num_keys + a.key_start[r];
  int* const rpos = rpos_all[wave];
  float* const rslope = rslope_all[wave];
  const int key = 32 * (wave & 1) + (lane & 31);
  for (int round = 0; round < rounds; ++round) {
    const int nvalid = it.left > 0 ? min(kSub, it.cur.len - it.j0) : 0, b0 = nvalid ? it.cur.pos + it.j0 : 0;
    const bool have = 32 * (wave & 1) < nvalid;
    u32x4 kh[D / 16], kl[D / 16];
    float acc[2] = {0.f, 0.f};
    if (have) load_keys<D, IL>(k_ptr(a.k_pool, it.cur, g, it.j0 + min(key, nvalid - 1), D), h2, kh);
    if (KM == kKeysNope && round == 0) {  // the first wait: angle rows (and the first query rows) in LDS for all
      wait_copies();
      __syncthreads();
    }
    if (have && ROT) {
      // Local-position keys turn by their record's position, the others by that of their 32-key block and a row's.
      if (lane < D / 2) turn_all[wave][lane] = rope_cs(LOCAL ? it.cur.pos : b0 + 32 * (wave & 1), rev);
      wait_reads();
      rotate_keys_split<D, KM, IL>(kh, kl, h2, turn_all[wave], [&](int t) {
        return *reinterpret_cast<const f32x4*>(trows + (lane & 31) * D + 4 * ((t / 2) ^ (lane & 15)));
      });
      wait_reads();
    }
    const auto compute = [&](int row0, const uint16_t* tq, const float* nl) {
      const int rows = min(kStepRows, row_end - row0);
      const int qmin = token_of(row0, a.group_magic) + shift, qmax = token_of(row0 + rows - 1, a.group_magic) + shift;
      if (!have || (a.causal && b0 > qmax)) return;
      const bool masked = (a.causal && b0 + kSub - 1 > qmin) || rows < kStepRows;
      if (ALIBI || masked) {
        if (lane < kStepRows) {
          const int src = row0 + lane, tok = token_of(src, a.group_magic);
          rpos[lane] = lane >= rows ? INT32_MIN : a.causal || ALIBI ? tok + shift : INT32_MAX;
          if (ALIBI) rslope[lane] = natural_slope(a, g * a.group + src - tok * a.group);
        }
        wait_reads();
      }
      const TileOperands<D> op(again(lane));
      f32x16 s = f32x16{};
      bf16x8 fh[2] = {op.row(tq, 0, 0)}, fl[2];
      if (ROT) fl[0] = op.row(tq + kStepRows * D, 0, 0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        if (k + 1 < D / 16) {
          fh[(k + 1) & 1] = op.row(tq, 0, k + 1);
          if (ROT) fl[(k + 1) & 1] = op.row(tq + kStepRows * D, 0, k + 1);
        }
        if (ROT) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fl[k & 1], as_bf16x8(kh[k]), s, 0, 0, 0);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fh[k & 1], as_bf16x8(kl[k]), s, 0, 0, 0);
        }
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fh[k & 1], as_bf16x8(kh[k]), s, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(nl + 8 * q4 + 4 * h2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 8 * q4 + 4 * h2 + e;
          s[4 * q4 + e] =
              fmaf(s[4 * q4 + e], a.scale_log2, ALIBI ? biased(rslope[row], b0 + key - rpos[row], x[e]) : x[e]);
        }
      }
      if (masked) {
        const int p = a.causal ? b0 + key : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = p <= rpos[8 * (i >> 2) + 4 * h2 + (i & 3)] ? s[i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i & 1] += fast_exp2(s[i]);
    };
    // The first rows lie in buffer 0 at the start of every round.
    for (int row0 = row_begin; row0 < row_end; row0 += 2 * kStepRows) {
      const int other = row0 + kStepRows, third = row0 + 2 * kStepRows;
      wait_copies();
      __syncthreads();
      if (other < row_end) fetch(other, tq1, nl1);
      compute(row0, tq0, nl0);
      if (other < row_end) {
        wait_copies();
        __syncthreads();
        // what comes next into buffer 0: the third step, or the next round's first
        if (third < row_end)
          fetch(third, tq0, nl0);
        else if (round + 1 < rounds)
          fetch(row_begin, tq0, nl0);
        compute(other, tq1, nl1);
      } else if (round + 1 < rounds && row0 != row_begin) {
        __syncthreads();
        fetch(row_begin, tq0, nl0);
      }
    }
    if (have) {
      const int at = it.base + it.j0 + key;
      const float sum = xor32_sum(acc[0] + acc[1]);
      if (h2 == 0 && key < nvalid && at < room) part[at] = sum;
    }
    it.skip(2);
  }
  wait_copies();
}

// Partial sums of the row splits and KV heads added up in their order.  Keys behind the table's last one are left alone.
__global__ __launch_bounds__(256) void sum_weights(WeightArgs a) {
  __shared__ int total[4];
  const int r = blockIdx.y, tid = threadIdx.x;
  int n = 0;
  for (int k = a.chunk_start[r] + tid; k < a.chunk_start[r + 1]; k += 256) n += a.chunks[k].len;
  n = wave_incl_scan(n);
  if ((tid & 63) == 63) total[tid >> 6] = n;
  __syncthreads();
  n = min(total[0] + total[1] + total[2] + total[3], min(a.key_start[r + 1], a.num_keys) - a.key_start[r]);
  for (int j = blockIdx.x * 256 + tid; j < n; j += gridDim.x * 256) {
    const int64_t at = (int64_t)a.key_start[r] + j;
    float w = 0.f;
    for (int p = 0; p < a.row_splits * a.hkv; ++p) w += a.ws_part[(int64_t)p * a.num_keys + at];
    a.weights[at] = a.weights_in ? fmaf(a.decay, a.weights_in[at], w) : w;
  }
}

// Weights of one new token per request: S = Q K^T of 16 keys and one KV head's queries at a time, a key in lane % 16.
// Rotated queries lie in LDS, kTokenRows rows at a time.
//   FEW (groups of up to kFewHeads query heads, keys that turn): products of 32-bit operands, 4 heads by 4 keys by 1
//     element, the lanes' quarters taking a quarter of the elements each; two swaps of halves add them up and leave one
//     head's score to a lane.  Nothing is split, and no rows of zeros are multiplied.
//   Otherwise 16x16x32 products of bf16 in two parts (ALiBi keys: one, exact), query heads 4 (lane / 16) + 0..3 of a group
//     of 16 in a lane's registers.
//   64 requests of 16384 keys, us, 4x4x1 against 16x16x32: groups of 4 278 / 382, of 7 198 / 211, of 8 395 / 431, of 16
//   167 / 130.
//   HS = 1: workgroup (key split, request); a wave takes 16 keys of each 64-key tile for all KV heads, whose angles it
//     forms once.
//   HS = 4: workgroup (16 keys of every tile of a key split, request); its waves share the KV heads and add up their sums
//     through LDS.  For batches whose tiles alone would leave CUs without work: a wave then waits for a quarter of the
//     loads.
// The next head's keys (or the next tile's first) are copied to LDS during a head's products, whole rows at a time: loads
// in the operands' layout touch 64 places of 16 bytes each and took 235 us for the same 2.1 GB by themselves, when all of
// them hit the first cache.  Bound there by the copies, which pass the L2s (253 us without the products), and close behind
// by rotation and products (234 us with copies of the same few rows).
//
// SORT: requests that share chunks list them in orders of their own.  The records of a request (up to kSortRecords) are
// walked in the order in which they are stored, and the workgroups of one key split of all requests run on one XCD: they
// then read the same part of the store at about the same time.  Every key's sum is its own, so results do not depend on
// the order.
constexpr int kFewHeads = 8;
constexpr int kTokenRows = 32, kTokenGroups = 16;  // query rows, and groups of up to 16 of one KV head, held in LDS
constexpr int kSortRecords = 256;
struct SortedRecord {
  int64_t koff;
  int32_t len, pos, kst, base;  // base: index of its first key among the request's keys
};
struct SortedTable {
  SortedRecord rec[kSortRecords] __attribute__((aligned(16)));
  uint32_t key[kSortRecords] __attribute__((aligned(16)));
  int tiles[kSortRecords];  // tiles of the records up to and with this one
  int wave_sum[4];

  // Sum of x over the threads before this one, and over all.
  __device__ int before(int x, int& total) {
    const int tid = threadIdx.x, incl = wave_incl_scan(x);
    __syncthreads();
    if ((tid & 63) == 63) wave_sum[tid >> 6] = incl;
    __syncthreads();
    int sum = incl - x;
    for (int w = 0; w < tid >> 6; ++w) sum += wave_sum[w];
    total = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    return sum;
  }
  // 256 threads; n <= kSortRecords records in units of 128 KiB of the store, table order within a unit.
  __device__ void build(const lazy_chunk_t* table, int count, int tk) {
    const int t = threadIdx.x;
    lazy_chunk_t c = {};
    if (t < count) c = table[t];
    int all;
    const int base = before(t < count ? c.len : 0, all);
    const uint32_t own = t < count ? (uint32_t)(c.k_offset >> 16) << 8 | (uint32_t)t : 0xffffffffu;
    key[t] = own;
    __syncthreads();
    int rank = 0;
    for (int j = 0; j < count; j += 4) {
      const u32x4 o = *reinterpret_cast<const u32x4*>(key + j);
      rank += (o[0] < own) + (o[1] < own) + (o[2] < own) + (o[3] < own);
    }
    if (t < count) rec[rank] = {c.k_offset, c.len, c.pos_offset, c.k_stride, base};
    __syncthreads();
    const int mine = t < count ? (rec[t].len + tk - 1) / tk : 0;
    tiles[t] = before(mine, all) + mine;
    __syncthreads();
  }
};
// A request's 64-key tiles, record after record of its sorted table, with the index of each record's first key among the
// request's keys.
struct SortedIter {
  const SortedTable* table;
  int i, j0, left, base;
  Rec cur;
  __device__ void load() {
    const SortedRecord r = table->rec[i];
    cur.koff =
        (int64_t)((uint64_t)(uint32_t)uniform((int)((uint64_t)r.koff >> 32)) << 32 | (uint32_t)uniform((int)r.koff));
    cur.len = uniform(r.len);
    cur.pos = uniform(r.pos);
    cur.kst = uniform(r.kst);
    base = uniform(r.base);
  }
  __device__ void start(const SortedTable* t, int n, int split, int splits) {
    table = t;
    const int total = n > 0 ? uniform(t->tiles[n - 1]) : 0;
    const int lo = (int)((int64_t)total * split / splits), hi = (int)((int64_t)total * (split + 1) / splits);
    left = hi - lo;
    i = j0 = base = 0;
    cur = {};
    if (left <= 0) return;
    int a = 0, b = n - 1;  // the first record whose tiles reach past lo
    while (a < b) {
      const int mid = (a + b) >> 1;
      if (uniform(t->tiles[mid]) > lo)
        b = mid;
      else
        a = mid + 1;
    }
    i = a;
    load();
    j0 = (lo - (uniform(t->tiles[i]) - (cur.len + kSub - 1) / kSub)) * kSub;
  }
  __device__ void next() {
    --left;
    j0 += kSub;
    if (left <= 0 || j0 < cur.len) return;
    j0 = 0;
    do {  // tiles are left, so a record with keys lies ahead
      ++i;
      load();
    } while (cur.len == 0);
  }
};

// Half a wave's (W = 32) or half a row pair's (W = 16) sums of x, and of y in the other half.
template <int W>
__device__ __forceinline__ float add_halves(float x, float y) {
  const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
  const auto z = W == 32 ? __builtin_amdgcn_permlane32_swap(a, b, false, false)
                         : __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return __uint_as_float(z[0]) + __uint_as_float(z[1]);
}

template <int D, int KMI, int HS, bool SORT, bool FEW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3))) void weigh_token(WeightArgs a) {
  constexpr int KM = keys_of(KMI);
  constexpr bool ALIBI = KM == kKeysAlibi, ROT = !ALIBI, LOCAL = KM == kKeysLocal, IL = interleaved_of(KMI);
  constexpr int QLD = D + kPad, H = D / 64, TPR = D / 16;
  constexpr int PARTS = ROT ? 2 : 1, FLD = D + 4;
  static_assert(ROT || !FEW);
  __shared__ uint16_t q[FEW ? 2 * kTokenRows * FLD : PARTS * kTokenRows * QLD] __attribute__((aligned(16)));
  float* const qf = reinterpret_cast<float*>(q);
  __shared__ float nlse[kTokenGroups * 16] __attribute__((aligned(16)));
  __shared__ float rslope[ALIBI ? kTokenGroups * 16 : 4] __attribute__((aligned(16)));
  __shared__ float2 qcs[D / 2];
  __shared__ float sums[2][4][16];
  // Angles of a wave's 16 keys: those of its first key, and of positions 0 .. 15 (rows 4 banks apart).  In 64 bits for
  // every key and pair they took a seventh of the time.
  constexpr int RLD = D + 4;
  __shared__ uint16_t tiles[4 * 16 * D] __attribute__((aligned(16)));  // a wave's 16 keys of one head
  __shared__ float2 base_all[4][D / 2] __attribute__((aligned(16)));
  __shared__ float rows16[KM == kKeysNope ? 16 * RLD : 4] __attribute__((aligned(16)));
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, kq = lane >> 4;
  int r = blockIdx.y, split = HS == 1 ? blockIdx.x : blockIdx.x >> 2;
  const int sub = HS == 1 ? wave : blockIdx.x & 3;
  if (SORT) {  // the splits' order, an eighth of it for each XCD
    const int id = blockIdx.x + gridDim.x * blockIdx.y, total = gridDim.x * gridDim.y, per = total >> 3;
    const int at = id < per << 3 ? (id & 7) * per + (id >> 3) : id;
    split = at / (int)gridDim.y;
    r = at - split * (int)gridDim.y;
  }
  // Loaded once: the compiler cannot know that the weights do not lie over them.
  const int qpos = uniform(a.q_pos0[r]), k0 = uniform(a.key_start[r]), room = uniform(a.key_start[r + 1]) - k0;
  const int c0 = a.chunk_start[r], c1 = a.chunk_start[r + 1];
  if (ROT && tid < D / 2) {
    qcs[tid] = rope_cs(a.rotate_q ? qpos : 0, revolutions(a, tid));
  }
  const double own_rev = ROT ? revolutions(a, lane % (D / 2)) : 0.0;
  if (KM == kKeysNope) {
    static_assert(256 % (D / 2) == 0, "a thread's entries share one pair");
    for (int e = tid; e < 16 * (D / 2); e += 256)
      *reinterpret_cast<float2*>(rows16 + e / (D / 2) * RLD + 2 * (e % (D / 2))) = rope_cs(e / (D / 2), own_rev);
  }
  const int per_head = (a.group + 15) / 16, groups = a.hkv * per_head, per_group = min(a.group, 16);
  const int most = min(kTokenGroups, kTokenRows / per_group);
  uint16_t* const tile = tiles + wave * 16 * D;
  // All groups of query heads over the tiles from it0 on.
  const auto walk = [&](const auto& it0) {
    for (int g0 = 0; g0 < groups; g0 += most) {
      const int ng = min(most, groups - g0);
      __syncthreads();
      for (int e = tid; e < ng * per_group * TPR; e += 256) {
        const int row = e / TPR, t0 = 8 * (e % TPR), grp = g0 + row / per_group;
        const int in = min((grp % per_head) * 16 + row % per_group, a.group - 1);
        const int64_t src = (int64_t)r * a.hq + (grp / per_head) * a.group + in;
        u32x4 lo, hi;
        load_pairs<D, IL>(a.q + src * D, t0, lo, hi);
        if (a.lse[src] == -INFINITY) lo = hi = u32x4{};
        uint16_t* const to = q + row * QLD + t0;
        if (ROT) {
          float yl[8], yh[8];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            rotate_by(element(lo, k), element(hi, k), qcs[t0 + k], yl[k], yh[k]);
          if (FEW) {
            float* const f = qf + row * FLD + t0;
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
              *reinterpret_cast<f32x4*>(f + k) = f32x4{yl[k], yl[k + 1], yl[k + 2], yl[k + 3]};
              *reinterpret_cast<f32x4*>(f + D / 2 + k) = f32x4{yh[k], yh[k + 1], yh[k + 2], yh[k + 3]};
            }
            continue;
          }
          u32x4 rest;
          split8(yl, lo, rest);
          *reinterpret_cast<u32x4*>(to + kTokenRows * QLD) = rest;
          split8(yh, hi, rest);
          *reinterpret_cast<u32x4*>(to + kTokenRows * QLD + D / 2) = rest;
        }
        *reinterpret_cast<u32x4*>(to) = lo;
        *reinterpret_cast<u32x4*>(to + D / 2) = hi;
      }
      for (int e = tid; e < ng * 16; e += 256) {  // rows past a group's end: exp2(score - inf) = 0
        const int grp = g0 + e / 16, in = (grp % per_head) * 16 + e % 16, h = (grp / per_head) * a.group + in;
        const float lse = in < a.group ? a.lse[(int64_t)r * a.hq + h] : -INFINITY;
        nlse[e] = lse == -INFINITY ? -INFINITY : -lse * lse_scale(KM);
        if (ALIBI) rslope[e] = in < a.group ? natural_slope(a, h) : 0.f;
      }
      __syncthreads();
      // A wave's groups: first, first + step, ...
      const int first = HS == 1 ? 0 : wave, step = HS;
      const float* const prior = g0 > 0 ? a.weights : a.weights_in;
      const float fade = g0 > 0 ? 1.f : a.decay;
      const auto fetch = [&](const auto& t, int k) {
        const uint16_t* const from = k_ptr(a.k_pool, t.cur, (g0 + k) / per_head, t.j0, D);
        const int last = t.cur.len - 1 - t.j0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const int row = (64 * i + lane) / (D / 8), chunk = (64 * i + lane) % (D / 8) ^ swizzle<D>(row);
          copy_async(from + (uint32_t)(min(16 * sub + row, last) * D + 8 * chunk), tile + 512 * i);
        }
      };
      const uint16_t* const qrow = q + min(col, per_group - 1) * QLD + 8 * kq;
      const float* const frow = qf + 8 * kq;
      auto it = it0, ahead = it0;
      int k = first, kf = first, parity = 0;
      float sum = 0.f, old = 0.f;
      float2 cs[H][8];
      const auto fetch_next = [&] {
        if (ahead.left <= 0) return;
        fetch(ahead, kf);
        kf += step;
        if (kf >= ng) {
          kf = first;
          ahead.next();
        }
      };
      const auto begin = [&] {
        const int key = it.j0 + 16 * sub + col, at = it.base + key;
        sum = old = 0.f;
        if (prior && key < it.cur.len && at < room) old = prior[k0 + at];
        if (ROT) {
          float2* const base = base_all[wave];
          if (lane < D / 2) base[lane] = rope_cs(LOCAL ? it.cur.pos : it.cur.pos + it.j0 + 16 * sub, own_rev);
          wait_reads();
#pragma unroll
          for (int s = 0; s < H; ++s)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const int t = 32 * s + 8 * kq + e;
              const f32x4 x = *reinterpret_cast<const f32x4*>(base + t);
              f32x4 y = {1.f, 0.f, 1.f, 0.f};
              if (!LOCAL) y = *reinterpret_cast<const f32x4*>(rows16 + col * RLD + 2 * t);
#pragma unroll
              for (int i = 0; i < 2; ++i)
                cs[s][e + i] = LOCAL ? make_float2(x[2 * i], x[2 * i + 1])
                                     : make_float2(fmaf(x[2 * i], y[2 * i], -(x[2 * i + 1] * y[2 * i + 1])),
                                                   fmaf(x[2 * i + 1], y[2 * i], x[2 * i] * y[2 * i + 1]));
            }
        }
      };
      const auto finish = [&] {
        const int key = it.j0 + 16 * sub + col, at = it.base + key;
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (HS > 1) {  // the waves' sums, in their order; two buffers, so one barrier a tile
          if (kq == 0) sums[parity][wave][col] = sum;
          __syncthreads();
          if (wave == 0) sum = (sums[parity][0][col] + sums[parity][1][col]) + (sums[parity][2][col] + sums[parity][3][col]);
          parity ^= 1;
        }
        if (a.causal && it.cur.pos + key > qpos) sum = 0.f;
        if ((HS == 1 || wave == 0) && kq == 0 && key < it.cur.len && at < room)
          a.weights[k0 + at] = prior ? fmaf(fade, old, sum) : sum;
        it.next();
      };
      const auto consume = [&] {
        u32x4 raw[H][2];
        wait_copies();
#pragma unroll
        for (int s = 0; s < H; ++s) {
          const int c = 4 * s + kq;
          raw[s][0] = *reinterpret_cast<const u32x4*>(tile + tile_at<D>(col, IL ? 2 * c : c));
          raw[s][1] = *reinterpret_cast<const u32x4*>(tile + tile_at<D>(col, IL ? 2 * c + 1 : D / 16 + c));
        }
        if (k == first) begin();
        wait_reads();
        fetch_next();
        if constexpr (FEW) {
          float yl[H][8], yh[H][8];
#pragma unroll
          for (int s = 0; s < H; ++s) {
            u32x4 lo = raw[s][0], hi = raw[s][1];
            if (IL) deinterleave8(raw[s][0], raw[s][1], lo, hi);
#pragma unroll
            for (int e = 0; e < 8; ++e) rotate_by(element(lo, e), element(hi, e), cs[s][e], yl[s][e], yh[s][e]);
          }
          for (int m = 0; m < per_group; m += 4) {
            const float* const at = frow + (k * per_group + min(m + (lane & 3), per_group - 1)) * FLD;
            f32x4 s4[2] = {f32x4{}, f32x4{}};
#pragma unroll
            for (int s = 0; s < H; ++s)
#pragma unroll
              for (int e = 0; e < 8; e += 4) {
                const f32x4 fl = *reinterpret_cast<const f32x4*>(at + 32 * s + e);
                const f32x4 fh = *reinterpret_cast<const f32x4*>(at + D / 2 + 32 * s + e);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  s4[0] = __builtin_amdgcn_mfma_f32_4x4x1f32(fl[i], yl[s][e + i], s4[0], 0, 0, 0);
                  s4[1] = __builtin_amdgcn_mfma_f32_4x4x1f32(fh[i], yh[s][e + i], s4[1], 0, 0, 0);
                }
              }
            s4[0] += s4[1];
            const float x = add_halves<32>(s4[0][0], s4[0][2]), y = add_halves<32>(s4[0][1], s4[0][3]);
            sum += fast_exp2(fmaf(add_halves<16>(x, y), a.scale_log2, nlse[16 * k + m + kq]));
          }
        } else {
          u32x4 kh[2 * H], kl[2 * H];
#pragma unroll
          for (int s = 0; s < H; ++s) {
            u32x4 lo = raw[s][0], hi = raw[s][1];
            if (IL) deinterleave8(raw[s][0], raw[s][1], lo, hi);
            if (ROT) {
              float yl[8], yh[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) rotate_by(element(lo, e), element(hi, e), cs[s][e], yl[e], yh[e]);
              split8(yl, lo, kl[s]);
              split8(yh, hi, kl[s + H]);
            }
            kh[s] = lo;
            kh[s + H] = hi;
          }
          f32x4 s4 = f32x4{};
#pragma unroll
          for (int s = 0; s < 2 * H; ++s) {
            const uint16_t* at = qrow + k * per_group * QLD + 32 * s;
            const bf16x8 fh = as_bf16x8(*reinterpret_cast<const u32x4*>(at));
            if (ROT) {
              const bf16x8 fl = as_bf16x8(*reinterpret_cast<const u32x4*>(at + kTokenRows * QLD));
              s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fl, as_bf16x8(kh[s]), s4, 0, 0, 0);
              s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fh, as_bf16x8(kl[s]), s4, 0, 0, 0);
            }
            s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fh, as_bf16x8(kh[s]), s4, 0, 0, 0);
          }
          {
            f32x4 x = *reinterpret_cast<const f32x4*>(nlse + 16 * k + 4 * kq);
            if (ALIBI) {
              const f32x4 sl = *reinterpret_cast<const f32x4*>(rslope + 16 * k + 4 * kq);
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = biased(sl[e], it.cur.pos + it.j0 + 16 * sub + col - qpos, x[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s4[e] = fmaf(s4[e], a.scale_log2, x[e]);
          }
          sum += (fast_exp2(s4[0]) + fast_exp2(s4[1])) + (fast_exp2(s4[2]) + fast_exp2(s4[3]));
        }
        k += step;
        if (k >= ng) {
          k = first;
          finish();
        }
      };
      if (first < ng) {
        fetch_next();
        while (it.left > 0) consume();
      } else {
        while (it.left > 0) finish();
      }
    }
  };
  if constexpr (SORT) {
    __shared__ SortedTable table;
    if (c1 - c0 <= kSortRecords) {
      table.build(a.chunks + c0, c1 - c0, kSub);
      SortedIter it;
      it.start(&table, c1 - c0, split, a.splits);
      walk(it);
      return;
    }
  }
  KeyIter it;
  it.start(a.chunks, c0, c1, split, a.splits);
  walk(it);
}

// Selection: a radix select of the b-th largest score, 11, 11 and 10 bits at a time, and an ordered compaction.  Scores
// are compared as integers in their order: NaN lowest, -0 like 0, protected keys above all.
//
// A workgroup of 1024 threads holds up to 35840 scores in LDS, so that a request of so many keys is read once and selected
// in one launch (select_request).  Longer requests are cut into slices of 16384 keys, one workgroup each: select_slices
// counts one digit a launch, leaving every slice's counts in the workspace, and the next launch (and the writing one)
// adds them up; nothing has to be cleared and no workgroup waits for another.
//
// One workgroup's passes are bound by its CU's vector instructions (64 lanes a clock: 33068 keys times one instruction is
// 0.2 us) and by LDS atomics on the same address (weights of a few octaves share their top bits).  So every pass does the
// least for a score: no bounds (the tail is filled up with the lowest score, which is never picked before a key), the
// first digit counted while the scores arrive, protected keys marked afterwards, passes that few scores concern skip
// whole waves, and every bin has two counters, one for every other lane (one counter: 3.5 us more).  33068 keys 22 us;
// 260 thousand in 16 slices 31 us in four launches, of which each chains loads, LDS passes and a sum over the slices'
// counts (slices of 8192 keys: 16% longer, and 65% for eight such requests).
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;
constexpr int kSlice = 16384, kMostResident = 35840;
__device__ __forceinline__ uint32_t score_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0 : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t with_digit(uint32_t prefix, int digit, int pass) {
  return prefix | (uint32_t)digit << (pass == 0 ? 21 : pass == 1 ? 10 : 0);
}

// x is in its register here: a load is not moved to a conditional use behind it, one of several in flight not put off.
template <class T>
__device__ __forceinline__ void loaded(T& x) {
  asm volatile("" : "+v"(x));
}

template <int CAP>
struct SelectSmem {
  uint32_t score[CAP] __attribute__((aligned(16)));
  int hist[2 * kBins] __attribute__((aligned(16)));  // two counters a digit
  int wave_sum[2 * kSelectWaves] __attribute__((aligned(8)));
  int digit, need;
};

constexpr int kBatch = 4;  // scores a thread has in flight
template <int CAP>
__device__ __forceinline__ void clear_counts(SelectSmem<CAP>& sm) {
  reinterpret_cast<u32x4*>(sm.hist)[threadIdx.x] = u32x4{0, 0, 0, 0};
  static_assert(2 * kBins == 4 * kSelectThreads);
  __syncthreads();
}

// Scores of keys j0 .. j0 + count - 1 (count <= CAP) of a request of n, filled up to a multiple of the workgroup's
// threads, and with COUNT their first digits.
template <bool COUNT, int CAP>
__device__ __forceinline__ int load_scores(SelectSmem<CAP>& sm, const float* w, int j0, int count, int n, int sink,
                                           int recent) {
  static_assert(CAP % kSelectThreads == 0);
  constexpr int U = 12;  // loads a thread has in flight
  const int tid = threadIdx.x, filled = (count + kSelectThreads - 1) & ~(kSelectThreads - 1);
  if (COUNT) clear_counts(sm);
  for (int base = 0; base < filled; base += U * kSelectThreads) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = w[j0 + min(base + u * kSelectThreads + tid, count - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) loaded(x[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (base + u * kSelectThreads >= filled) break;
      const int i = base + u * kSelectThreads + tid;
      uint32_t s = score_of(x[u]);
      if (base + (u + 1) * kSelectThreads > count && i >= count) s = 0;
      sm.score[i] = s;
      if (COUNT) atomicAdd(&sm.hist[2 * (s >> 21) + (tid & 1)], 1);
    }
  }
  __syncthreads();
  const auto protect = [&](int i) {
    if (COUNT) {
      atomicAdd(&sm.hist[2 * (sm.score[i] >> 21) + (tid & 1)], -1);
      atomicAdd(&sm.hist[2 * (kBins - 1) + (tid & 1)], 1);
    }
    sm.score[i] = 0xffffffffu;
  };
  const int head = min(max(0, sink - j0), count), tail = max(head, n - recent - j0);
  for (int i = tid; i < head; i += kSelectThreads) protect(i);
  for (int i = tail + tid; i < count; i += kSelectThreads) protect(i);
  __syncthreads();
  return filled;
}

// Counts the digits of pass 1 or 2.
template <int CAP>
__device__ __forceinline__ void count_digits(SelectSmem<CAP>& sm, int filled, uint32_t prefix, int pass) {
  const int tid = threadIdx.x, shift = pass == 1 ? 10 : 0;
  const uint32_t width = pass == 1 ? 1u << 21 : 1u << 10;
  clear_counts(sm);
  for (int base = 0; base < filled; base += kBatch * kSelectThreads) {
    uint32_t s[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e)
      s[e] = sm.score[min(base + e * kSelectThreads, filled - kSelectThreads) + tid] - prefix;
#pragma unroll
    for (int e = 0; e < kBatch; ++e)
      if (base + e * kSelectThreads < filled && s[e] < width) atomicAdd(&sm.hist[2 * (s[e] >> shift) + (tid & 1)], 1);
  }
  __syncthreads();
}
// This thread's two bins, from the largest digit down.
template <int CAP>
__device__ __forceinline__ int2 own_bins(const SelectSmem<CAP>& sm, int pair) {
  const u32x4 x = reinterpret_cast<const u32x4*>(sm.hist)[pair];
  return make_int2((int)(x[0] + x[1]), (int)(x[2] + x[3]));
}

// The digit in which the need-th largest score lies and its rank among those with that digit.  count: this thread's bins
// 2047 - 2 tid and 2046 - 2 tid.
template <int CAP>
__device__ __forceinline__ void find_digit(SelectSmem<CAP>& sm, const int (&count)[2], int need) {
  const int tid = threadIdx.x, wave = tid >> 6;
  const int sum = count[0] + count[1], incl = wave_incl_scan(sum);
  if ((tid & 63) == 63) sm.wave_sum[wave] = incl;
  __syncthreads();
  int before = incl - sum;
  for (int w = 0; w < wave; ++w) before += sm.wave_sum[w];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (before < need && need <= before + count[e]) {
      sm.digit = kBins - 1 - 2 * tid - e;
      sm.need = need - before;
    }
    before += count[e];
  }
  __syncthreads();
}

// Writes the indices of the scores above the threshold and of the first `need` equal to it, in order; `above` and
// `equal` of either come before this workgroup's.  Every wave counts, then writes, a part of its own.
template <int CAP>
__device__ __forceinline__ void write_kept(SelectSmem<CAP>& sm, int j0, int filled, uint32_t threshold, int need,
                                           int above, int equal, int32_t* out) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int per = filled / kSelectWaves;  // a multiple of 64
  const uint32_t* const mine = sm.score + wave * per + lane;
  int na = 0, ne = 0;
  for (int i = 0; i < per; i += 64 * kBatch) {
    uint32_t s[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) s[e] = mine[min(i + 64 * e, per - 64)];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) loaded(s[e]);
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      if (i + 64 * e >= per) break;
      na += __builtin_popcountll(__ballot(s[e] > threshold));
      ne += __builtin_popcountll(__ballot(s[e] == threshold));
    }
  }
  if (lane == 0) *reinterpret_cast<int2*>(&sm.wave_sum[2 * wave]) = make_int2(na, ne);
  __syncthreads();
  na = above;
  ne = equal;
  for (int w = 0; w < wave; ++w) {
    na += sm.wave_sum[2 * w];
    ne += sm.wave_sum[2 * w + 1];
  }
  const int first = j0 + wave * per + lane;
  const auto before = [](uint64_t m) {  // lanes below this one in a mask
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
  };
  for (int i = 0; i < per; i += 64 * kBatch) {
    uint32_t s[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) s[e] = mine[min(i + 64 * e, per - 64)];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) loaded(s[e]);
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      if (i + 64 * e >= per) break;
      const uint64_t ma = __ballot(s[e] > threshold), me = __ballot(s[e] == threshold);
      if (me) {  // rare
        const int re = ne + before(me);
        if (s[e] > threshold || (s[e] == threshold && re < need)) out[na + before(ma) + min(re, need)] = first + i + 64 * e;
      } else if (s[e] > threshold) {
        out[na + min(ne, need) + before(ma)] = first + i + 64 * e;
      }
      na += __builtin_popcountll(ma);
      ne += __builtin_popcountll(me);
    }
  }
}

struct SelectArgs {
  const float* weights;
  const int32_t* key_start;
  const int32_t* key_count;
  const int32_t* kept_start;
  int32_t* kept;
  int32_t* ws;  // [batch][slices] of SliceWork (long requests)
  int sink, recent, slices;
};
// A slice's counts of each pass's digits; the digits found so far, the rank left, and earlier slices' scores above them.
struct SliceWork {
  int hist[3][kBins];
  uint32_t prefix;
  int need, above, unused;
};

__device__ __forceinline__ bool trivial_selection(const SelectArgs& a, int n, int b, int o0) {
  if (b >= n) {
    for (int i = blockIdx.x * kSelectThreads + threadIdx.x; i < b; i += gridDim.x * kSelectThreads)
      a.kept[o0 + i] = i < n ? i : -1;
    return true;
  }
  return b <= 0;
}

template <int CAP>
__global__ __launch_bounds__(kSelectThreads) void select_request(SelectArgs a) {
  __shared__ SelectSmem<CAP> sm;
  const int r = blockIdx.y, tid = threadIdx.x;
  const int k0 = a.key_start[r], room = a.key_start[r + 1] - k0;
  const int n = min(a.key_count ? max(0, min(a.key_count[r], room)) : room, CAP);
  const int o0 = a.kept_start[r], b = a.kept_start[r + 1] - o0;
  if (trivial_selection(a, n, b, o0)) return;
  const int filled = load_scores<true>(sm, a.weights + k0, 0, n, n, a.sink, a.recent);
  uint32_t prefix = 0;
  int need = b;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    if (pass > 0) count_digits(sm, filled, prefix, pass);
    const int2 x = own_bins(sm, kSelectThreads - 1 - tid);
    const int c[2] = {x.y, x.x};
    find_digit(sm, c, need);
    prefix = with_digit(prefix, sm.digit, pass);
    need = sm.need;
    __syncthreads();
  }
  write_kept(sm, 0, filled, prefix, need, 0, 0, a.kept + o0);
}

// Launch `pass` of a long request's selection: 0 to 2 count a digit, 3 writes.
template <int PASS>
__global__ __launch_bounds__(kSelectThreads) void select_slices(SelectArgs a) {
  __shared__ SelectSmem<kSlice> sm;
  __shared__ int before_s[2];
  const int r = blockIdx.y, w = blockIdx.x, tid = threadIdx.x;
  const int k0 = a.key_start[r], room = a.key_start[r + 1] - k0;
  const int most = (int)min((int64_t)a.slices * kSlice, (int64_t)INT32_MAX);
  const int n = min(a.key_count ? max(0, min(a.key_count[r], room)) : room, most);
  const int o0 = a.kept_start[r], b = a.kept_start[r + 1] - o0;
  if (b >= n || b <= 0) {
    if (PASS == 3) trivial_selection(a, n, b, o0);
    return;
  }
  SliceWork* const all = reinterpret_cast<SliceWork*>(a.ws) + (int64_t)r * a.slices;
  const int used = (n - 1) / kSlice + 1;
  if (w >= used) return;
  const int j0 = w * kSlice, count = min(kSlice, n - j0);
  const float* const scores = a.weights + k0 + j0;
  SliceWork& own = all[w];
  // Passes 1 and 2 look at every score once: in registers, loaded while the counts are added up.
  constexpr bool ONCE = PASS == 1 || PASS == 2;
  constexpr int PER = kSlice / kSelectThreads;
  float x[PER];
  int filled = 0;
  if constexpr (ONCE) {
#pragma unroll
    for (int u = 0; u < PER; ++u) x[u] = scores[min(u * kSelectThreads + tid, count - 1)];
    clear_counts(sm);
  } else {
    filled = load_scores<PASS == 0>(sm, a.weights + k0, j0, count, n, a.sink, a.recent);
  }
  uint32_t prefix = 0;
  int need = b;
  if constexpr (PASS > 0) {  // the digit counted last, from every slice's counts
    if (tid < 2) before_s[tid] = PASS > 1 && tid == 0 ? own.above : 0;
    if (PASS > 1) {
      prefix = own.prefix;
      need = own.need;
    }
    int c[2] = {0, 0}, earlier[2] = {0, 0};
    const int b1 = kBins - 1 - 2 * tid;
    constexpr int B = 16;
    for (int v0 = 0; v0 < used; v0 += B) {
      int2 y[B];
#pragma unroll
      for (int v = 0; v < B; ++v)
        y[v] = *reinterpret_cast<const int2*>(&all[min(v0 + v, used - 1)].hist[PASS - 1][b1 - 1]);
#pragma unroll
      for (int v = 0; v < B; ++v) {
        c[0] += v0 + v < used ? y[v].y : 0;
        c[1] += v0 + v < used ? y[v].x : 0;
        earlier[0] += v0 + v < w ? y[v].y : 0;
        earlier[1] += v0 + v < w ? y[v].x : 0;
      }
    }
    find_digit(sm, c, need);
    const int digit = sm.digit;
    prefix = with_digit(prefix, digit, PASS - 1);
    need = sm.need;
    const int above = wave_incl_scan((b1 > digit ? earlier[0] : 0) + (b1 - 1 > digit ? earlier[1] : 0));
    if ((tid & 63) == 63 && above) atomicAdd(&before_s[0], above);
    if (b1 == digit || b1 - 1 == digit) before_s[1] = b1 == digit ? earlier[0] : earlier[1];
    __syncthreads();
  }
  if (PASS < 3) {
    if (PASS > 0) {
      if (tid == 0) {
        own.prefix = prefix;
        own.need = need;
        own.above = before_s[0];
      }
      const uint32_t width = PASS == 1 ? 1u << 21 : 1u << 10;
      const int head = a.sink - j0, tail = n - a.recent - j0;
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int i = u * kSelectThreads + tid;
        const uint32_t d = (i < head || i >= tail ? 0xffffffffu : score_of(x[u])) - prefix;
        if (i < count && d < width) atomicAdd(&sm.hist[2 * (d >> (PASS == 1 ? 10 : 0)) + (tid & 1)], 1);
      }
      __syncthreads();
    }
    *reinterpret_cast<int2*>(&own.hist[PASS][2 * tid]) = own_bins(sm, tid);
  } else {
    write_kept(sm, j0, filled, prefix, need, before_s[0], before_s[1], a.kept + o0);
  }
}

// Gather of kept keys: workgroup (64 kept keys, KV head, request).  The records that hold them are found by prefix sums
// over the request's table, 256 records at a time.  Bound by memory: 64 requests, 2048 of 16.4K keys each, 255 us for 1.08
// GB (4.2 TB/s; a large copy 4.7).
constexpr int kGather = 64;
template <int D, int TURN, bool LOCAL, bool IL>
__global__ __launch_bounds__(256) void gather_keys(CompactArgs a) {
  __shared__ int ends[256], wsum[4];
  __shared__ int64_t ksrc[kGather], vsrc[kGather];
  __shared__ int turn[kGather];
  __shared__ double freq[D / 2];
  const int r = blockIdx.z, g = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int o0 = a.kept_start[r], count = a.kept_start[r + 1] - o0, i0 = blockIdx.x * kGather;
  if (i0 >= count) return;
  const int i = i0 + tid;  // threads 0 .. 63: one kept key each
  int want = tid < kGather && i < count ? a.kept[o0 + i] : -1;
  const int asked = want;
  if (tid < kGather) ksrc[tid] = -1;
  if (TURN && tid < D / 2) freq[tid] = revolutions(a, tid);
  const lazy_chunk_t dst = a.dst[r];
  int base = 0;
  for (int c0 = a.chunk_start[r]; c0 < a.chunk_start[r + 1]; c0 += 256) {
    const int nrec = min(256, a.chunk_start[r + 1] - c0);
    const int incl = wave_incl_scan(tid < nrec ? a.chunks[c0 + tid].len : 0);
    if (lane == 63) wsum[wave] = incl;
    __syncthreads();
    int before = base;
    for (int w = 0; w < wave; ++w) before += wsum[w];
    ends[tid] = before + incl;
    base += wsum[0] + wsum[1] + wsum[2] + wsum[3];
    __syncthreads();
    if (want >= 0 && want < base) {
      int lo = 0, hi = nrec - 1;  // the first record that ends past the key
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > want)
          hi = mid;
        else
          lo = mid + 1;
      }
      const lazy_chunk_t c = a.chunks[c0 + lo];
      const int j = want - (ends[lo] - c.len);
      ksrc[tid] = c.k_offset + ((int64_t)g * c.k_stride + j) * D;
      vsrc[tid] = c.v_offset + ((int64_t)g * c.v_stride + j) * D;
      turn[tid] = TURN == 2 ? i - j : LOCAL ? c.pos_offset : c.pos_offset + j;
      want = -1;
    }
  }
  __syncthreads();
  if (a.weights_out && g == 0 && tid < kGather && i < count)
    a.weights_out[o0 + i] =
        ksrc[tid] >= 0 && asked < a.key_start[r + 1] - a.key_start[r] ? a.weights[a.key_start[r] + asked] : 0.f;
  constexpr int TPR = D / 16;
  const int t0 = 8 * (tid % TPR);
  for (int row = tid / TPR; row < kGather; row += 256 / TPR) {
    const int at = i0 + row;
    if (at >= count || ksrc[row] < 0 || at >= dst.k_stride || at >= dst.v_stride) continue;
    const uint16_t* ks = a.k_pool + ksrc[row];
    const uint16_t* vs = a.v_pool + vsrc[row];
    uint16_t* kd = a.k_out + dst.k_offset + ((int64_t)g * dst.k_stride + at) * D;
    uint16_t* vd = a.v_out + dst.v_offset + ((int64_t)g * dst.v_stride + at) * D;
    if (TURN) {
      u32x4 lo, hi;
      load_pairs<D, IL>(ks, t0, lo, hi);
      float yl[8], yh[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        rotate_by(element(lo, e), element(hi, e), rope_cs(turn[row], freq[t0 + e]), yl[e], yh[e]);
      store_pairs<D, IL>(kd, t0, yl, yh);
    } else {
      reinterpret_cast<u32x4*>(kd + 2 * t0)[0] = reinterpret_cast<const u32x4*>(ks + 2 * t0)[0];
      reinterpret_cast<u32x4*>(kd + 2 * t0)[1] = reinterpret_cast<const u32x4*>(ks + 2 * t0)[1];
    }
    reinterpret_cast<u32x4*>(vd + 2 * t0)[0] = reinterpret_cast<const u32x4*>(vs + 2 * t0)[0];
    reinterpret_cast<u32x4*>(vd + 2 * t0)[1] = reinterpret_cast<const u32x4*>(vs + 2 * t0)[1];
  }
}

template <int D, int KMI>
hipError_t prompt_mode(const WeightArgs& a, int max_kv_len, hipStream_t s) {
  const int blocks = (a.total_q + kPrepTokens - 1) / kPrepTokens, more = keys_of(KMI) == kKeysNope ? kAngleBlocks<D> : 0;
  if (blocks + more) prepare_queries<D, KMI><<<blocks + more, 256, 0, s>>>(a, blocks);
  weigh_prompt<D, KMI><<<dim3(a.splits * a.row_splits, a.hkv, a.batch), 256, 0, s>>>(a);
  sum_weights<<<dim3(ceil_div(max_kv_len, 256), a.batch), 256, 0, s>>>(a);
  return hipGetLastError();
}
template <int D, int KMI, bool FEW>
hipError_t token_heads(const WeightArgs& a, hipStream_t s) {
  if (a.head_split)
    weigh_token<D, KMI, 4, false, FEW><<<dim3(4 * a.splits, a.batch), 256, 0, s>>>(a);
  else if (a.sort_records)
    weigh_token<D, KMI, 1, true, FEW><<<dim3(a.splits, a.batch), 256, 0, s>>>(a);
  else
    weigh_token<D, KMI, 1, false, FEW><<<dim3(a.splits, a.batch), 256, 0, s>>>(a);
  return hipGetLastError();
}
template <int D, int KMI>
hipError_t token_mode(const WeightArgs& a, hipStream_t s) {
  if constexpr (keys_of(KMI) != kKeysAlibi)
    if (a.group <= kFewHeads) return token_heads<D, KMI, true>(a, s);
  return token_heads<D, KMI, false>(a, s);
}

template <int D, int TURN, bool LOCAL>
void compact_mode(const CompactArgs& a, dim3 grid, bool interleaved, hipStream_t s) {
  if (interleaved)
    gather_keys<D, TURN, LOCAL, true><<<grid, 256, 0, s>>>(a);
  else
    gather_keys<D, TURN, LOCAL, false><<<grid, 256, 0, s>>>(a);
}
template <int D>
void compact_dim(const CompactArgs& a, dim3 grid, int turn, bool local_keys, bool interleaved, hipStream_t s) {
  if (turn == 0)
    gather_keys<D, 0, false, false><<<grid, 256, 0, s>>>(a);
  else if (turn == 2)
    compact_mode<D, 2, true>(a, grid, interleaved, s);
  else if (local_keys)
    compact_mode<D, 1, true>(a, grid, interleaved, s);
  else
    compact_mode<D, 1, false>(a, grid, interleaved, s);
}

}  // namespace

#define LAZY_KEY_MODES(CALL)                                              \
  if (alibi) return CALL(kKeysAlibi);                                     \
  if (local_keys) {                                                       \
    if (interleaved) return CALL(kKeysLocal | kInterleaved);              \
    return CALL(kKeysLocal);                                              \
  }                                                                       \
  if (interleaved) return CALL(kKeysNope | kInterleaved);                 \
  return CALL(kKeysNope);

hipError_t launch_prefill_weights(const WeightArgs& a, int head_dim, bool local_keys, bool interleaved, bool alibi,
                                  int max_kv_len, hipStream_t s) {
#define CALL(KM) (head_dim == 64 ? prompt_mode<64, KM>(a, max_kv_len, s) : prompt_mode<128, KM>(a, max_kv_len, s))
  LAZY_KEY_MODES(CALL)
#undef CALL
}

hipError_t launch_decode_weights(const WeightArgs& a, int head_dim, bool local_keys, bool interleaved, bool alibi,
                                 hipStream_t s) {
#define CALL(KM) (head_dim == 64 ? token_mode<64, KM>(a, s) : token_mode<128, KM>(a, s))
  LAZY_KEY_MODES(CALL)
#undef CALL
}

size_t select_workspace(int batch, int max_kv_len) {
  return max_kv_len <= kMostResident ? 0 : sizeof(SliceWork) * (size_t)batch * (size_t)ceil_div(max_kv_len, kSlice);
}

// The least instance that holds the longest request: LDS decides how many workgroups share a CU.
hipError_t launch_select(const float* weights, const int32_t* key_start, const int32_t* key_count,
                         const int32_t* kept_start, int batch, int max_kv_len, int sink, int recent, int32_t* kept,
                         void* workspace, hipStream_t s) {
  SelectArgs a = {weights, key_start, key_count, kept_start, kept, static_cast<int32_t*>(workspace), sink, recent, 0};
  const dim3 one(1, batch);
  if (max_kv_len <= kSlice) {
    select_request<kSlice><<<one, kSelectThreads, 0, s>>>(a);
  } else if (max_kv_len <= kMostResident) {
    select_request<kMostResident><<<one, kSelectThreads, 0, s>>>(a);
  } else {
    a.slices = (int)ceil_div(max_kv_len, kSlice);
    const dim3 grid(a.slices, batch);
    select_slices<0><<<grid, kSelectThreads, 0, s>>>(a);
    select_slices<1><<<grid, kSelectThreads, 0, s>>>(a);
    select_slices<2><<<grid, kSelectThreads, 0, s>>>(a);
    select_slices<3><<<grid, kSelectThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs& a, int head_dim, int batch, int max_kept, int turn, bool local_keys,
                          bool interleaved, hipStream_t s) {
  const dim3 grid(ceil_div(max_kept, kGather), a.hkv, batch);
  if (head_dim == 64)
    compact_dim<64>(a, grid, turn, local_keys, interleaved, s);
  else
    compact_dim<128>(a, grid, turn, local_keys, interleaved, s);
  return hipGetLastError();
}

}  // namespace lazy
