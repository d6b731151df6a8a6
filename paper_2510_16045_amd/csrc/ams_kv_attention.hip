// Attention over the 4-bit KV cache.
//
//   S[r, j] = softmax_scale * q[r] . k[j],  O[r] = sum_j exp(S[r, j] - max) v[j] / sum_j exp(S[r, j] - max)
//
// with k and v as the cache holds them (fp16 values), sums and statistics in fp32.  The heads / kv_heads query heads that read one
// kv head are rows of one problem: row r of a sequence is token r / R of its query rows and head r % R of the kv head's R.
//
// stream_kernel: one read of the cache.  A workgroup takes 16 QT rows and a piece of the keys, its four wavefronts take every fourth
// step of 32 keys, straight from memory to registers: K's words become the A operand of S^T = K q^T, the result tile lies as the B
// operand of O^T = V^T P^T wants it (a lane has the same four keys of a tile in both), V's words become its A operand.  No LDS, no
// barrier before the end, where the wavefronts' partial sums are joined.
//
// Pieces: the host knows neither lengths nor (with row starts) how many rows a sequence has, so every workgroup works out the same
// split from them: the steps of all sequences over the workgroups that fill the chip, rounded up, is the length of a piece.  A piece
// of a sequence that has several leaves (max, sum, O) in the workspace, and join_kernel adds those up in the order of the pieces.
#include "ams_kv.h"

#include <float.h>

#include <algorithm>

namespace ams_kv {

constexpr int kStep = 32;         // keys of a wavefront's step
constexpr int kStreamWaves = 4;
constexpr int kMinPiece = 4;      // steps of a piece: one for each wavefront
constexpr float kLift = 8.0f;     // exponents of P are raised by this: below it P keeps fp16's full precision over 2^-22 of the largest
constexpr float kSlack = 7.0f;    // how far (log2) a score may pass the running maximum before that is raised: 2^(8 + 7) is in fp16

struct AttentionArgs {
  View v;
  const uint16_t* q;
  uint16_t* out;
  float *lse, *part;  // part: [slot][kv head][row of the tile][D + 2]
  int64_t q_stride, q_head, out_stride, out_head, lse_stride;
  float scale2;  // softmax_scale * log2(e)
  int group;     // R
  int heads_pieces;  // pieces that the sequences of one kv head are cut into, about; 0: none is cut
  int causal, window, vec;
};

// What one sequence contributes: rows, row tiles and steps of keys.
struct Extent {
  int start, n, len, lo, row_tiles, steps;  // lo: first key (a multiple of kStep) that any row may see
};
template <int ROWS>
__device__ __forceinline__ Extent extent_of(const AttentionArgs& a, int b) {
  Extent e;
  e.start = row_start(a.v, b);
  e.n = max(row_start(a.v, b + 1) - e.start, 0);
  e.len = kv_len(a.v, b);
  const int first = e.len - e.n;  // position of the first row
  e.lo = a.window > 0 ? max(first + 1 - a.window, 0) & ~(kStep - 1) : 0;
  e.row_tiles = (int)(((int64_t)e.n * a.group + ROWS - 1) / ROWS);
  e.steps = e.row_tiles > 0 ? max((e.len - e.lo + kStep - 1) / kStep, 0) : 0;
  return e;
}

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i, 64);
  return x;
}
__device__ __forceinline__ int wave_prefix(int x) {  // inclusive
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int y = __shfl_up(x, i, 64);
    if (lane_id() >= i) x += y;
  }
  return x;
}

// Steps of a piece: the same for every workgroup of a call.
template <int ROWS>
__device__ __forceinline__ int piece_steps(const AttentionArgs& a) {
  if (a.heads_pieces == 0) return 0x7FFFFFFF;
  int64_t total = 0;
  for (int b = 0; b < a.v.batch; b += 64)
    if (b + lane_id() < a.v.batch) {
      const Extent e = extent_of<ROWS>(a, b + lane_id());
      total += (int64_t)e.row_tiles * e.steps;
    }
  total = wave_sum(total);
  const int64_t piece = (total + a.heads_pieces - 1) / a.heads_pieces;
  return (int)min(max((piece + kMinPiece - 1) / kMinPiece * kMinPiece, (int64_t)kMinPiece), (int64_t)0x7FFFFF00);
}

// A piece of work: rows of tile `row_tile` of sequence b, piece `piece` of `pieces`; slot: where the first piece of the tile leaves its
// result.  With JOIN an item is a row tile.
struct Item {
  int b, row_tile, piece, pieces, slot;
};
template <int ROWS, bool JOIN>
__device__ __forceinline__ bool find_item(const AttentionArgs& a, int per_piece, int item, Item* out) {
  int items = 0, slots = 0;
  for (int b0 = 0; b0 < a.v.batch; b0 += 64) {
    const int b = b0 + lane_id();
    int pieces = 0, tiles = 0;
    if (b < a.v.batch) {
      const Extent e = extent_of<ROWS>(a, b);
      tiles = e.row_tiles;
      pieces = tiles > 0 ? max(1, (int)(((int64_t)e.steps + per_piece - 1) / per_piece)) : 0;
    }
    const int mine = JOIN ? tiles : tiles * pieces, taken = pieces > 1 ? tiles * pieces : 0;
    const int end = wave_prefix(mine) + items, slot_end = wave_prefix(taken) + slots;
    const unsigned long long past = __ballot(end > item);
    if (past) {
      const int at = __builtin_ctzll(past);
      const int local = item - (__shfl(end, at, 64) - __shfl(mine, at, 64));
      pieces = __shfl(pieces, at, 64);
      out->b = b0 + at;
      out->pieces = pieces;
      out->row_tile = JOIN ? local : local / pieces;
      out->piece = JOIN ? 0 : local % pieces;
      out->slot = __shfl(slot_end, at, 64) - __shfl(taken, at, 64) + out->row_tile * pieces;
      return true;
    }
    items = __shfl(end, 63, 64);
    slots = __shfl(slot_end, 63, 64);
  }
  return false;
}

__device__ __forceinline__ h8 join_halves(h4 a, h4 b) { return h8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }

// The lowest and highest key (one past) that the row at `position` may see.
__device__ __forceinline__ int key_end(const AttentionArgs& a, int len, int position) { return a.causal ? min(len, position + 1) : len; }
__device__ __forceinline__ int key_begin(const AttentionArgs& a, int position) { return a.window > 0 ? max(position + 1 - a.window, 0) : 0; }

// Words and scales of two tiles of a step.
template <int D, int G>
struct StepData {
  Lane<D> k[2], v[2];
  Scales<D / G> sk[2];
  Scales<4 * D / G> sv[2];
  bool held[2];  // the table names a page for the tile
  __device__ __forceinline__ void load(const AttentionArgs& a, int b, int head, int step, int lane) {
    constexpr int RUNS = D / G, CODES = 8 * D, SCALES = kTile * RUNS * 2;
#pragma unroll
    for (int t = 0; t < 2; t++) {
      const int tile = 2 * step + t;
      const uint8_t* block = block_of(a.v, b, tile, head);
      held[t] = block != nullptr;
      if (!block) block = a.v.pages;  // read, and left out
      const uint8_t* const kc = block + tile % a.v.page_tiles * CODES;
      const uint8_t* const ks = block + 2 * a.v.codes + tile % a.v.page_tiles * SCALES;
      k[t].load(kc, lane);
      v[t].load(kc + a.v.codes, lane);
      sk[t].load(ks + (lane & 15) * RUNS * 2);
      sv[t].load(ks + a.v.scales + (lane >> 4) * RUNS * 8);
    }
  }
};

__device__ __forceinline__ bool not_finite(_Float16 x) { return (__builtin_bit_cast(uint16_t, x) & 0x7C00) == 0x7C00; }

// Runs of V that stand for NaN take part in a step's products as zeros where not every row sees every key of the step; here the rows
// that do see one get the NaN.
template <int D, int G, int QT>
__device__ __forceinline__ void nan_of_seen_keys(const StepData<D, G>& x, int first_key, const int (&begin)[QT], const int (&end)[QT], f4 (&o)[D / 16][QT]) {
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4 * D / G; i++) any |= not_finite(x.sv[0].s[i]) || not_finite(x.sv[1].s[i]);
  if (!__ballot(any)) return;
#pragma unroll
  for (int run = 0; run < D / G; run++) {
    uint32_t keys = 0;  // of the step, whose run stands for NaN
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const unsigned long long lanes = __ballot(x.held[u] && not_finite(x.sv[u].s[4 * run + j]));
#pragma unroll
        for (int g = 0; g < 4; g++) keys |= (uint32_t)(lanes >> 16 * g & 1) << (16 * u + 4 * g + j);
      }
#pragma unroll
    for (int t = 0; t < QT; t++) {
      const int from = min(max(begin[t] - first_key, 0), 32), to = min(max(end[t] - first_key, 0), 32);
      const uint32_t seen = (uint32_t)((1ull << to) - 1) & ~(uint32_t)((1ull << from) - 1);
      if (keys & seen) {
#pragma unroll
        for (int d = run * G / 16; d < (run + 1) * G / 16; d++) o[d][t] = f4{NAN, NAN, NAN, NAN};
      }
    }
  }
}

template <int D, int G, int QT>
__global__ __launch_bounds__(64 * kStreamWaves) void stream_kernel(AttentionArgs a) {
  constexpr int ROWS = 16 * QT, RUNS = D / G, DT = D / 16, KB = D / 32;
  const int tid = threadIdx.x, wave = tid >> 6, lane = lane_id(), g = lane >> 4, col = lane & 15;
  const int head = blockIdx.x % a.v.kv_heads;
  Item it;
  const int per_piece = piece_steps<ROWS>(a);
  if (!find_item<ROWS, false>(a, per_piece, blockIdx.x / a.v.kv_heads, &it)) return;
  const Extent e = extent_of<ROWS>(a, it.b);
  const int rows = e.n * a.group, row0 = it.row_tile * ROWS;
  // this lane's rows: one in each column tile
  h8 q[KB][QT];
  int begin[QT], end[QT];
#pragma unroll
  for (int t = 0; t < QT; t++) {
    const int r = row0 + 16 * t + col;
    const bool there = r < rows;
    const int token = there ? r / a.group : 0, position = e.len - e.n + token;
    begin[t] = there ? key_begin(a, position) : 0;
    end[t] = there ? key_end(a, e.len, position) : 0;
    const uint16_t* src = a.q + (int64_t)(e.start + token) * a.q_stride + (int64_t)(head * a.group + (there ? r % a.group : 0)) * a.q_head + 8 * g;
#pragma unroll
    for (int i = 0; i < KB; i++) {
      u4 x = {0, 0, 0, 0};
      if (there) {
        if (a.vec) {
          x = *(const u4*)(src + 32 * i);
        } else {
#pragma unroll
          for (int j = 0; j < 4; j++) x[j] = src[32 * i + 2 * j] | (uint32_t)src[32 * i + 2 * j + 1] << 16;
        }
      }
      q[i][t] = __builtin_bit_cast(h8, x);
    }
  }
  // the piece's steps that some row of the tile sees, and those in which every row sees every key
  const int first_token = row0 / a.group, last_token = min(row0 + ROWS, rows) - 1;
  const int p_first = e.len - e.n + first_token, p_last = e.len - e.n + last_token / a.group;
  const int step_end = (key_end(a, e.len, p_last) + kStep - 1) / kStep, step_begin = key_begin(a, p_first) / kStep;
  const int from = max((int)min((int64_t)it.piece * per_piece, (int64_t)0x7FFFFFF) + e.lo / kStep, step_begin);
  const int to = min((int)min((int64_t)(it.piece + 1) * per_piece, (int64_t)0x7FFFFFF) + e.lo / kStep, step_end);
  const int whole_begin = key_begin(a, p_last), whole_end = key_end(a, e.len, p_first);

  f4 o[DT][QT];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; t++) {
    m[t] = -INFINITY, l[t] = 0;
#pragma unroll
    for (int d = 0; d < DT; d++) o[d][t] = f4{0, 0, 0, 0};
  }
  for (int step = from + wave; step < to; step += kStreamWaves) {
    StepData<D, G> x;
    x.load(a, it.b, head, step, lane);
    f4 s[2][QT];
#pragma unroll
    for (int u = 0; u < 2; u++) {
#pragma unroll
      for (int t = 0; t < QT; t++) s[u][t] = f4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < KB; i++) {
        const h8 k = restore_k(x.k[u].w[i], x.sk[u].s[32 * i / G]);
#pragma unroll
        for (int t = 0; t < QT; t++) s[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[i][t], s[u][t], 0, 0, 0);
      }
    }
    const bool whole = step * kStep >= whole_begin && (step + 1) * kStep <= whole_end && x.held[0] && x.held[1];
    h8 p[QT];
#pragma unroll
    for (int t = 0; t < QT; t++) {
      if (!whole) {
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const int key = step * kStep + 16 * u + 4 * g + i;
            if (key < begin[t] || key >= end[t] || !x.held[u]) s[u][t][i] = -INFINITY;
          }
      }
      float top = m[t];
#pragma unroll
      for (int u = 0; u < 2; u++)
#pragma unroll
        for (int i = 0; i < 4; i++) top = fmaxf(top, s[u][t][i] * a.scale2);
      // the maximum is raised only where a score passes it by more than the slack: then for all lanes that share the row
      if (__ballot(top > m[t] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float less = top > m[t] ? __builtin_amdgcn_exp2f(m[t] - top) : 1.0f;
        m[t] = top;
        l[t] *= less;
#pragma unroll
        for (int d = 0; d < DT; d++) o[d][t] *= less;
      }
      const float sub = m[t] == -INFINITY ? 0.0f : m[t] - kLift;
#pragma unroll
      for (int u = 0; u < 2; u++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][t][i], a.scale2, -sub));
          l[t] += v;
          p[t][4 * u + i] = (_Float16)v;
        }
    }
#pragma unroll
    for (int i = 0; i < KB; i++) {
      const int run = 32 * i / G * 4;
      h4 va[2], vb[2];
#pragma unroll
      for (int u = 0; u < 2; u++) {
        h4 sv = {x.sv[u].s[run], x.sv[u].s[run + 1], x.sv[u].s[run + 2], x.sv[u].s[run + 3]};
        if (!whole) {  // a masked key's P is 0, and 0 times what it holds has to be
#pragma unroll
          for (int j = 0; j < 4; j++)
            if (not_finite(sv[j])) sv[j] = (_Float16)0;
        }
        restore_v(x.v[u].w[i], sv, &va[u], &vb[u]);
      }
#pragma unroll
      for (int t = 0; t < QT; t++) {
        o[2 * i][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join_halves(va[0], va[1]), p[t], o[2 * i][t], 0, 0, 0);
        o[2 * i + 1][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join_halves(vb[0], vb[1]), p[t], o[2 * i + 1][t], 0, 0, 0);
      }
    }
    if (!whole) nan_of_seen_keys<D, G, QT>(x, step * kStep, begin, end, o);
  }

  // The wavefronts' results are joined in their order; eight d-tiles of one column tile at a time go through LDS.
  constexpr int AT_ONCE = DT < 8 ? DT : 8;
  __shared__ __align__(16) f4 parts[kStreamWaves][AT_ONCE][64];
  __shared__ float tops[kStreamWaves][ROWS], sums[kStreamWaves][ROWS];
#pragma unroll
  for (int t = 0; t < QT; t++) {
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
    if (g == 0) tops[wave][16 * t + col] = m[t], sums[wave][16 * t + col] = l[t];
  }
  __syncthreads();
  const bool alone = it.pieces == 1;
  float* const part = a.part + ((int64_t)(it.slot + it.piece) * a.v.kv_heads + head) * ROWS * (D + 2);
#pragma unroll
  for (int t = 0; t < QT; t++) {
    const int r = row0 + 16 * t + col;
    float top = -INFINITY, sum = 0, by[kStreamWaves];
#pragma unroll
    for (int w = 0; w < kStreamWaves; w++) top = fmaxf(top, tops[w][16 * t + col]);
#pragma unroll
    for (int w = 0; w < kStreamWaves; w++) {
      const float mine = tops[w][16 * t + col];
      by[w] = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
      sum += sums[w][16 * t + col] * by[w];
    }
    const float scale = alone ? (sum > 0 || sum != sum ? 1.0f / sum : 0.0f) : 1.0f;
#pragma unroll
    for (int d0 = 0; d0 < DT; d0 += AT_ONCE) {
      __syncthreads();
#pragma unroll
      for (int d = 0; d < AT_ONCE; d++) parts[wave][d][lane] = o[d0 + d][t];
      __syncthreads();
      for (int d = wave; d < AT_ONCE; d += kStreamWaves) {
        f4 x = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kStreamWaves; w++) x += parts[w][d][lane] * by[w];
        if (r >= rows) continue;
        x *= scale;
        const int channel = 16 * (d0 + d) + 4 * g;
        if (alone) {
          uint16_t* const dst = a.out + (int64_t)(e.start + r / a.group) * a.out_stride + (int64_t)(head * a.group + r % a.group) * a.out_head + channel;
          const h4 y = {(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3]};
          if (a.vec) {
            *(h4*)dst = y;
          } else {
#pragma unroll
            for (int j = 0; j < 4; j++) ((_Float16*)dst)[j] = y[j];
          }
        } else {
          float* const dst = part + (16 * t + col) * (D + 2) + 2 + channel;
#pragma unroll
          for (int j = 0; j < 4; j++) dst[j] = x[j];
        }
      }
    }
    if (wave == 0 && g == 0 && r < rows) {
      if (!alone) {
        part[(16 * t + col) * (D + 2)] = top;
        part[(16 * t + col) * (D + 2) + 1] = sum;
      } else if (a.lse) {
        a.lse[(int64_t)(e.start + r / a.group) * a.lse_stride + head * a.group + r % a.group] = sum > 0 || sum != sum ? (top - kLift + __log2f(sum)) * 0.69314718056f : -INFINITY;
      }
    }
  }
}

// Adds up the pieces of a row tile that has several.  A wavefront takes rows of the tile, its lanes the channels.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void join_kernel(AttentionArgs a) {
  const int wave = threadIdx.x >> 6, lane = lane_id(), head = blockIdx.x % a.v.kv_heads;
  Item it;
  const int per_piece = piece_steps<ROWS>(a);
  if (!find_item<ROWS, true>(a, per_piece, blockIdx.x / a.v.kv_heads, &it) || it.pieces == 1) return;
  const Extent e = extent_of<ROWS>(a, it.b);
  const int rows = min(e.n * a.group - it.row_tile * ROWS, ROWS);
  const int64_t stride = (int64_t)a.v.kv_heads * ROWS * (D + 2);
  for (int i = wave; i < rows; i += 4) {
    const float* const part = a.part + ((int64_t)it.slot * a.v.kv_heads + head) * ROWS * (D + 2) + i * (D + 2);
    float top = -INFINITY, sum = 0, x[D / 64];
#pragma unroll
    for (int j = 0; j < D / 64; j++) x[j] = 0;
    for (int s = 0; s < it.pieces; s++) top = fmaxf(top, part[s * stride]);
    for (int s = 0; s < it.pieces; s++) {
      const float mine = part[s * stride], by = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
      sum += part[s * stride + 1] * by;
#pragma unroll
      for (int j = 0; j < D / 64; j++) x[j] += part[s * stride + 2 + 64 * j + lane] * by;
    }
    const int r = it.row_tile * ROWS + i;
    const float scale = sum > 0 || sum != sum ? 1.0f / sum : 0.0f;
    uint16_t* const dst = a.out + (int64_t)(e.start + r / a.group) * a.out_stride + (int64_t)(head * a.group + r % a.group) * a.out_head;
#pragma unroll
    for (int j = 0; j < D / 64; j++) dst[64 * j + lane] = __builtin_bit_cast(uint16_t, (_Float16)(x[j] * scale));
    if (a.lse && lane == 0)
      a.lse[(int64_t)(e.start + r / a.group) * a.lse_stride + head * a.group + r % a.group] = sum > 0 || sum != sum ? (top - kLift + __log2f(sum)) * 0.69314718056f : -INFINITY;
  }
}

// ---- launch ------------------------------------------------------------------------------------------
constexpr int kTargetGroups = 1024;  // workgroups that fill the chip

struct Plan {
  int qt, rows;
  int64_t row_tiles;    // at most so many over all sequences
  int64_t tile_steps;   // at most so many steps of one row tile
  int64_t pieces;       // heads_pieces
  size_t workspace;     // bytes that this many pieces need
};
Plan make_plan(const ams_kv_cache* c, int64_t rows, int heads, int64_t max_q_len, size_t workspace) {
  Plan p;
  const int R = heads / c->kv_heads;
  const int64_t most = (c->q_starts ? std::min(max_q_len > 0 ? max_q_len : rows, rows) : 1) * R;
  p.qt = most <= 16 ? 1 : most <= 32 || c->head_dim == 256 ? 2 : 4;
  p.rows = 16 * p.qt;
  p.row_tiles = c->q_starts ? rows * R / p.rows + c->batch : c->batch * (int64_t)((R + p.rows - 1) / p.rows);
  p.tile_steps = ((int64_t)c->table_width * c->page_size + kStep - 1) / kStep;
  const size_t slot = (size_t)c->kv_heads * p.rows * (c->head_dim + 2) * sizeof(float);
  p.pieces = std::max<int64_t>(kTargetGroups / c->kv_heads, 1);
  // sequences that are cut have fewer than twice as many pieces as all have on average
  if (p.tile_steps <= kMinPiece) p.pieces = 0;
  p.pieces = std::min<int64_t>(p.pieces, (int64_t)(std::min<size_t>(workspace, AMS_KV_WORKSPACE_BYTES) / slot / 2));
  p.workspace = 2 * (size_t)p.pieces * slot;
  return p;
}

}  // namespace ams_kv

using namespace ams_kv;

extern "C" {

int ams_kv_attention_workspace_bytes(const ams_kv_cache* cache, int64_t rows, int heads, int64_t max_q_len, size_t* bytes) {
  View v;
  if (!bytes) return AMS_ERR_NULL;
  if (const int rc = make_view(cache, rows, &v); rc != AMS_OK) return rc;
  if (heads < 1 || heads % cache->kv_heads || heads > AMS_KV_MAX_HEADS) return AMS_ERR_SHAPE;
  *bytes = make_plan(cache, rows, heads, max_q_len, SIZE_MAX).workspace;
  return AMS_OK;
}

int ams_kv_attention(const ams_kv_cache* cache, const uint16_t* Q, uint16_t* O, float* lse, int64_t rows, int heads, int64_t q_stride, int64_t q_head_stride,
                     int64_t o_stride, int64_t o_head_stride, int64_t lse_stride, float softmax_scale, int causal, int64_t window, int64_t max_q_len,
                     void* workspace, size_t workspace_bytes, void* stream) {
  AttentionArgs a;
  if (const int rc = make_view(cache, rows, &a.v); rc != AMS_OK) return rc;
  if (rows > 0 && (!Q || !O)) return AMS_ERR_NULL;
  if (heads < 1 || heads % cache->kv_heads || heads > AMS_KV_MAX_HEADS || window < 0 || (window > 0 && !causal) || max_q_len < 0 || !(softmax_scale > 0) || !(softmax_scale <= FLT_MAX)) return AMS_ERR_SHAPE;
  if (rows * (heads / cache->kv_heads) > AMS_KV_MAX_TOKENS) return AMS_ERR_SHAPE;
  if (!aligned(Q, 2) || !aligned(O, 2) || !aligned(lse, 4) || !aligned(workspace, 16)) return AMS_ERR_ALIGN;
  if (const int rc = device_status(); rc != AMS_OK) return rc;
  if (rows == 0 || cache->batch == 0) return AMS_OK;
  a.q = Q, a.out = O, a.lse = lse, a.part = (float*)workspace;
  a.q_stride = q_stride, a.q_head = q_head_stride, a.out_stride = o_stride, a.out_head = o_head_stride, a.lse_stride = lse_stride;
  a.scale2 = softmax_scale * 1.44269504089f;
  a.group = heads / cache->kv_heads;
  a.causal = causal != 0, a.window = (int)std::min<int64_t>(window, 0x3FFFFFFF);
  a.vec = aligned(Q, 16) && aligned(O, 8) && (q_stride | q_head_stride) % 8 == 0 && (o_stride | o_head_stride) % 4 == 0;
  const Plan p = make_plan(cache, rows, heads, max_q_len, workspace ? workspace_bytes : 0);
  a.heads_pieces = (int)p.pieces;
  const int64_t items = std::min(p.row_tiles + p.pieces, p.row_tiles * ((p.tile_steps + kMinPiece - 1) / kMinPiece + 1));
  const int64_t grid = items * cache->kv_heads, joins = p.row_tiles * cache->kv_heads;
  if (grid > 0x7FFFFFFF) return AMS_ERR_SHAPE;
  auto launch = [&](auto kernel, int64_t n) { hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(256), 0, (hipStream_t)stream, a); };
  dispatch(cache->head_dim, cache->scale_group, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    switch (p.qt) {
      case 1: launch(stream_kernel<D, G, 1>, grid); break;
      case 2: launch(stream_kernel<D, G, 2>, grid); break;
      default:
        if constexpr (D < 256) launch(stream_kernel<D, G, 4>, grid);  // 256 accumulators do not fit beside the rows
    }
    if (p.pieces == 0) return;
    switch (p.qt) {
      case 1: launch(join_kernel<D, 16>, joins); break;
      case 2: launch(join_kernel<D, 32>, joins); break;
      default: launch(join_kernel<D, 64>, joins); break;
    }
  });
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

}  // extern "C"
