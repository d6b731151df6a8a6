// Attention over the 4-bit KV cache: what its two kernels share.
//
//   S[r, j] = softmax_scale * q[r] . k[j],  O[r] = sum_j exp(S[r, j] - max) v[j] / sum_j exp(S[r, j] - max)
//
// with k and v as the cache holds them (fp16 values), sums and statistics in fp32.  The heads / kv_heads query heads that read one
// kv head are rows of one problem: row r of a sequence is token r / R of its query rows and head r % R of the kv head's R.
//
// Split of the work: the host knows neither lengths nor (with row starts) how many rows a sequence has, so every workgroup works it
// out from them.  tile_kernel's workgroups take a tile of rows each.  For stream_kernel the steps of all row tiles of a kv head are shared
// out among as many workgroups as fit on the chip at once:
//   where no tile has more than kUncutSteps, whole tiles;
//   where there are two shares or more for a tile, parts of one tile each, of up to so many steps that there are enough shares (8 sequences
//   of 2400 with 16 rows, 32 query and 8 kv heads: 37 us if shares cross tiles, 24 so; 16 of 3001 with 40 rows 30 and 28.5; 8 of 2000 with
//   4 rows 17 and 13; but 4 of 3000 11.7 and 12.4: the split takes longer to work out);
//   else, and for a tile alone, which has no other to cross into, equal shares of all steps, one tile after the other, which may begin and
//   end inside a tile; that a workgroup begins a tile counts as much as kTileSteps steps.
// Of a tile that lies in several shares every workgroup leaves its part (max, sum, O) in the workspace and counts itself in; the one that
// comes last adds all of them up, always in the same order, and clears the count.  Nobody waits for anybody.
#ifndef AMS_KV_ATTENTION_H_
#define AMS_KV_ATTENTION_H_

#include "ams_kv.h"

namespace ams_kv {

constexpr int kDeviceScope = 16;  // cache policy (sc1) of a buffer load or store that the whole device sees
constexpr int kStep = 32;         // keys of a wavefront's step
constexpr int kMinShare = 16;     // steps of a share (4 sequences of 3000, 8 kv heads: 8 or 16 11.5 us, 32 17.6)
constexpr int kTileSteps = 14;    // what it takes to begin a tile and to leave its result, in steps (32 ragged sequences of up to 8192, 8 kv heads: 8 42.8 us, 14 41.5, 24 42.3)
constexpr int kUncutSteps = 32;   // a tile of so many is not cut: joining its parts takes longer than its steps (64 of up to 1000, 4 kv heads: 32 or 64 11.2 us, 16 18.4)
constexpr int kMaxParts = 64;     // of a tile (one of 131071: at most 32 parts 54 us, 64 41, 128 42; 64 rows of it, one kv head: 64 52, 128 59)
constexpr int kNear = 8;          // parts of a tile that are added up first where there are many (64 rows of 131071, one kv head: 4 62 us, 8 52; 8 kv heads: 8 85, 16 90)
constexpr int kTrips = 2;         // one workgroup adds up all parts of a tile if it waits for them no more than so often
constexpr float kLift = 8.0f;     // exponents of P are raised by this: below it P keeps fp16's full precision over 2^-22 of the largest
constexpr float kSlack = 7.0f;    // how far (log2) a score may pass the running maximum before that is raised: 2^(8 + 7) is in fp16
constexpr float kFar = 1048576;   // maxima (log2) from which on exponents are differences of rounded products: below it a product that is not
                                  // rounded lies within 2^-5 of one that is, far above it further than fp16 reaches

struct AttentionArgs {
  View v;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  uint32_t* counts;  // [of tiles, of kNear shares of a tile][kv head][share in which they begin]
  float* parts;      // [kv head][2 share + (the tile begins in it)][row of the tile][max, sum, -, -, D values]
  int64_t q_stride, q_head, out_stride, out_head, lse_stride;
  float scale2;  // softmax_scale * log2(e)
  int group;     // R
  Divisor by_group;
  int shares;        // workgroups of one kv head
  int cut;           // whether a tile may lie in several
  int row_tiles;     // at most so many over all sequences, if row starts ascend
  int part_rows;     // rows of a tile in `parts`
  int causal, window, vec;
};

// What one sequence contributes: rows, row tiles and steps of keys.
struct Extent {
  int start, n, len, lo, row_tiles, steps;  // lo: first key (a multiple of kStep) that any row may see
};
template <int ROWS>
__device__ __forceinline__ Extent extent_of(const AttentionArgs& a, int b) {
  Extent e = {0, 0, 0, 0, 0, 0};
  if (b >= a.v.batch) return e;
  e.start = row_start(a.v, b);
  e.n = max(row_start(a.v, b + 1) - e.start, 0);
  e.len = kv_len(a.v, b);
  const int first = e.len - e.n;  // position of the first row
  e.lo = a.window > 0 ? max(first + 1 - a.window, 0) & ~(kStep - 1) : 0;
  e.row_tiles = (int)(((uint32_t)e.n * (uint32_t)a.group + ROWS - 1) / ROWS);
  e.steps = max((e.len - e.lo + kStep - 1) / kStep, 1);  // one also where there is no key: somebody has to say so
  return e;
}

// Sums over the lanes up to a lane's own: within rows of 16, then the rows'.  Every lane of the wavefront takes part.  Lane patterns of
// the adds themselves; trips through LDS, six at a time and two times on every workgroup's way to its first load, cost half a
// microsecond to a microsecond a call.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
  constexpr int kUp = 0x110, kRowEnd = 0x142, kHalfEnd = 0x143;  // n lanes up in a row; the end of the row before; of the first half
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kUp + 1, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kUp + 2, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kUp + 4, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kUp + 8, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kRowEnd, 0xA, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kHalfEnd, 0xC, 0xF, false);
  return x;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix(x), 63); }
// A lane's value and that of the lane 32 (16) further, in either order.
__device__ __forceinline__ f2 with_32(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return f2{__builtin_bit_cast(float, (unsigned)y[0]), __builtin_bit_cast(float, (unsigned)y[1])};
}
__device__ __forceinline__ f2 with_16(float x) {
  const auto y = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return f2{__builtin_bit_cast(float, (unsigned)y[0]), __builtin_bit_cast(float, (unsigned)y[1])};
}
__device__ __forceinline__ float larger(f2 x) { return fmaxf(x[0], x[1]); }
__device__ __forceinline__ float sum_of(f2 x) { return x[0] + x[1]; }

// Whether some lane's maximum is that large (rows that have seen no key yet have none).
__device__ __forceinline__ bool any_far(float top) { return __ballot(fabsf(top) >= kFar && top != -INFINITY) != 0; }
// x - top in log2, 0 for the score that the maximum `top` comes from: its product has been rounded as this one is.
__device__ __forceinline__ float below_top(float x, float scale2, float top) {
#pragma clang fp contract(off)
  const float y = x * scale2;
  return top == -INFINITY ? y : y - top;
}

// x, of which the compiler knows nothing: what follows from it is not worked out before it is needed and kept in registers.
__device__ __forceinline__ int hidden(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int of_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// How much a share is, and all row tiles together: in tiles that are not cut; in parts of one tile each, of which a step is `pieces`; or in
// steps with kTileSteps more for each tile.
struct Split {
  uint32_t per, total;
  float pieces;
  bool cut;
};
__device__ __forceinline__ uint32_t tile_cost(const Extent& e, const Split& split) {
  if (!split.cut) return 1;
  return split.pieces > 0 ? (uint32_t)((float)e.steps * split.pieces) + 1 : e.steps + kTileSteps;
}
template <int ROWS>
__device__ __forceinline__ Split split_of(const AttentionArgs& a, const Extent& first) {  // first: of the first 64 sequences
  uint32_t tiles = first.row_tiles, steps = first.row_tiles * first.steps, most = first.row_tiles > 0 ? first.steps : 0;
  for (int b0 = 64; b0 < a.v.batch; b0 += 64) {
    const Extent x = extent_of<ROWS>(a, b0 + lane_id());
    tiles = min(tiles + x.row_tiles, 1u << 25), steps += x.row_tiles * x.steps, most = max(most, x.row_tiles > 0 ? (uint32_t)x.steps : 0);
  }
  Split split = {1, 0, 0.0f, a.cut && __ballot(most > (uint32_t)kUncutSteps) != 0};
  const uint32_t shares = (uint32_t)a.shares;
  tiles = wave_sum(tiles), steps = wave_sum(steps);
  if (tiles > (uint32_t)a.row_tiles) return split;  // starts that do not ascend: there is no bound to the work, and the sums may wrap
  split.total = split.cut ? steps + tiles * kTileSteps : tiles;
  if (split.cut && tiles > 1 && 2 * tiles <= shares) {
    const float each = __builtin_amdgcn_rcpf((float)steps) * 0.9999f;  // rounds down: no more parts than shares
#pragma unroll 1
    for (uint32_t spare = tiles / 2;; spare = tiles) {  // shares that rounding up takes: half a part of a tile as a rule, one at most
      split.pieces = fminf((float)(shares - spare) * each, 1.0f / kMinShare);
      uint32_t parts = first.row_tiles * tile_cost(first, split);
      for (int b0 = 64; b0 < a.v.batch; b0 += 64) {
        const Extent x = extent_of<ROWS>(a, b0 + lane_id());
        parts += x.row_tiles * tile_cost(x, split);
      }
      split.total = wave_sum(parts);
      if (split.total <= shares || spare == tiles) return split;
    }
  }
  split.per = max((split.total + shares - 1) / shares, split.cut ? (uint32_t)kMinShare : 1u);
  return split;
}

// The row tile that the cost `at` of the whole falls on, where its own begins and how much it is.
struct Place {
  Extent e;
  int b, row_tile;
  uint32_t first, cost;
};
template <int ROWS>
__device__ __forceinline__ bool place_of(const AttentionArgs& a, Extent e, const Split& split, uint32_t at, Place* out) {  // e: of the first 64 sequences
  uint32_t before = 0;
  for (int b0 = 0; b0 < a.v.batch; b0 += 64) {
    if (b0 > 0) e = extent_of<ROWS>(a, b0 + lane_id());
    const uint32_t each = tile_cost(e, split), mine = e.row_tiles * each;
    const uint32_t end = wave_prefix(mine) + before;
    const unsigned long long past = __ballot(end > at);
    if (past) {
      const int lane = __builtin_ctzll(past);
      const uint32_t first = of_lane(end - mine, lane);
      out->b = b0 + lane;
      out->cost = of_lane(each, lane);
      out->row_tile = (at - first) / out->cost;
      out->first = first + out->row_tile * out->cost;
      out->e = {of_lane(e.start, lane), of_lane(e.n, lane), of_lane(e.len, lane), of_lane(e.lo, lane), of_lane(e.row_tiles, lane), of_lane(e.steps, lane)};
      return true;
    }
    before = of_lane(end, 63);
  }
  return false;
}

__device__ __forceinline__ h8 join_halves(u2 a, u2 b) { return __builtin_bit_cast(h8, u4{a[0], a[1], b[0], b[1]}); }

// Eight halfs; where rows are not 16-byte aligned half by half.
__device__ __forceinline__ u4 load_half8(const uint16_t* p, bool vec) {
  if (vec) return *(const u4*)p;
  u4 x;
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  return x;
}

// The lowest and highest key (one past) that the row at `position` may see.
__device__ __forceinline__ int key_end(const AttentionArgs& a, int len, int position) { return a.causal ? min(len, position + 1) : len; }
__device__ __forceinline__ int key_begin(const AttentionArgs& a, int position) { return a.window > 0 ? max(position + 1 - a.window, 0) : 0; }

// A row tile that lies in several shares.
struct Pending {
  int start, row0, rows, first, count;  // start: its sequence's first row; first: the first of the shares
};

__device__ __forceinline__ void store_out(const AttentionArgs& a, int start, int head, int r, int channel, f4 x) {
  const int token = (int)a.by_group.quotient((uint32_t)r);
  _Float16* const dst = (_Float16*)a.out + (int64_t)(start + token) * a.out_stride + (int64_t)(head * a.group + r - token * a.group) * a.out_head + channel;
  const h4 y = {(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3]};
  if (a.vec) {
    *(h4*)dst = y;
  } else {
#pragma unroll
    for (int j = 0; j < 4; j++) dst[j] = y[j];
  }
}
__device__ __forceinline__ void store_lse(const AttentionArgs& a, int start, int head, int r, float top, float sum) {
  if (!a.lse) return;
  const int token = (int)a.by_group.quotient((uint32_t)r);
  a.lse[(int64_t)(start + token) * a.lse_stride + head * a.group + r - token * a.group] = sum > 0 || sum != sum ? (top - kLift + __log2f(sum)) * 0.69314718056f : -INFINITY;
}

// Adds up the parts of a row tile.  D / 4 lanes take a row, four channels each; of the workgroup's groups of lanes as many take rows
// as there are (a power of two), U rows each at once, and the others share the parts of a row, P of them at once: U P parts of rows are
// asked for before the first is used.  The parts are those of every APARTth share from `from` on; the sum becomes the tile's result, or
// takes the place of the first of them.
template <int D, int THREADS, int U, int P, int APART = 1, bool RESULT = true>
__device__ __forceinline__ void join_parts(const AttentionArgs& a, const Pending& tile, __amdgpu_buffer_rsrc_t left, int head, float* lds, int from, int count) {
  constexpr int LANES = D / 4, GROUPS = THREADS / LANES;
  f4* const xs = (f4*)lds;                // [group][lane]
  f2* const stats = (f2*)(xs + THREADS);  // [group]
  const int group = threadIdx.x / LANES, c = threadIdx.x % LANES;
  const int rows = tile.rows;
  int takers = 1;  // groups that take rows
  while (takers < rows && takers < GROUPS) takers *= 2;
  const int sharers = GROUPS / takers, mine = group / takers;
  auto place = [&](int s, int i) { return ((2 * (from + s * APART) + (s == 0 && from == tile.first)) * a.part_rows + i) * (D + 4) * 4; };
  auto add = [](float& top, float& sum, f4& x, float part_top, float part_sum, f4 more) {
    const float most = fmaxf(top, part_top);
    const float less = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - most), by = part_top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(part_top - most);
    top = most;
    sum = sum * less + part_sum * by;
    x = x * less + more * by;
  };
#pragma unroll 1
  for (int i0 = 0; i0 < rows; i0 += takers * U) {
    float top[U], sum[U];
    f4 x[U];
#pragma unroll
    for (int u = 0; u < U; u++) top[u] = -INFINITY, sum[u] = 0, x[u] = f4{0, 0, 0, 0};
#pragma unroll 1
    for (int s0 = mine; s0 < count; s0 += sharers * P) {
      f4 part[U][P];
      f2 stat[U][P];
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int j = 0; j < P; j++) {
          const int s = s0 + j * sharers, i = i0 + u * takers + group % takers;
          const int at = s < count && i < rows ? place(s, i) : 0x7FFE0000;  // nothing is read there
          part[u][j] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(left, at + 16 + 16 * c, 0, kDeviceScope));
          stat[u][j] = __builtin_bit_cast(f2, __builtin_amdgcn_raw_buffer_load_b64(left, at, 0, kDeviceScope));
          if (s >= count) stat[u][j] = f2{-INFINITY, 0};
        }
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int j = 0; j < P; j++) add(top[u], sum[u], x[u], stat[u][j][0], stat[u][j][1], part[u][j]);
    }
    if (sharers > 1) {  // then every row has a taker, in its first turn
      xs[threadIdx.x] = x[0];
      if (c == 0) stats[group] = f2{top[0], sum[0]};
      __syncthreads();
      for (int j = 1; j < sharers && mine == 0; j++) add(top[0], sum[0], x[0], stats[j * takers + group][0], stats[j * takers + group][1], xs[(j * takers + group) * LANES + c]);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int i = i0 + u * takers + group % takers;
      if (mine > 0 || i >= rows) continue;
      if constexpr (RESULT) {
        store_out(a, tile.start, head, tile.row0 + i, 4 * c, x[u] * (sum[u] > 0 || sum[u] != sum[u] ? 1.0f / sum[u] : 0.0f));
        if (c == 0) store_lse(a, tile.start, head, tile.row0 + i, top[u], sum[u]);
      } else {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x[u]), left, place(0, i) + 16 + 16 * c, 0, kDeviceScope);
        if (c == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, f2{top[u], sum[u]}), left, place(0, i), 0, kDeviceScope);
      }
    }
  }
}

// The end of a workgroup whose share has `pending` tiles that lie in others too (only its first and its last can).  Every wavefront's
// stores have been acknowledged before the workgroup is counted in, and the parts are asked for after the count has come back; they go
// to the level of the memory system that all compute units share.  Where one workgroup would wait for memory more than kTrips
// times, the last of every kNear shares adds up theirs, and the last of those workgroups the sums: 64 rows of one sequence of 131071
// and one kv head 137 -> 52 us, with 8 kv heads 116 -> 84.  Where that rule says one, two would cost a second count: 16 sequences of
// 3001 with 40 rows 33 -> 40, one of 131071 with 4 rows 36 -> 38.
template <int D, int THREADS, int U, int P>
__device__ __forceinline__ void join_pending(const AttentionArgs& a, int pending, const Pending& first, const Pending& last, __amdgpu_buffer_rsrc_t left, int share, int head, float* lds, bool* all_there) {
  if (pending == 0) return;
  auto in_two = [](const Pending& tile) { return tile.rows * tile.count > kTrips * (THREADS / (D / 4)) * U * P; };
  auto count_in = [&](uint32_t* counts, int at, int of) {  // whether this workgroup is the last
    uint32_t* const counter = counts + head * a.shares + at;
    const bool is_last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)of - 1;
    if (is_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return is_last;
  };
  auto near = [&](const Pending& tile) { return max(share - tile.first, 0) / kNear * kNear; };  // the first of the shares that are added up together
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x < (unsigned)pending) {
    const Pending tile = threadIdx.x == 0 ? first : last;
    if (in_two(tile)) {
      const int at = near(tile), members = min(tile.count - at, kNear);
      all_there[threadIdx.x] = members < 2 || count_in(a.counts + a.shares * a.v.kv_heads, tile.first + at, members);
    } else {
      all_there[threadIdx.x] = count_in(a.counts, tile.first, tile.count);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i < pending; i++) {
    if (!all_there[i]) continue;
    const Pending tile = i == 0 ? first : last;
    if (!in_two(tile)) {
      join_parts<D, THREADS, U, P>(a, tile, left, head, lds, tile.first, tile.count);
      continue;
    }
    const int members = min(tile.count - near(tile), kNear), sums = (tile.count + kNear - 1) / kNear;
    if (members > 1) join_parts<D, THREADS, U, P, 1, false>(a, tile, left, head, lds, tile.first + near(tile), members);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) all_there[i] = count_in(a.counts, tile.first, sums);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (all_there[i]) join_parts<D, THREADS, U, P, kNear>(a, tile, left, head, lds, tile.first, sums);
  }
}

// ---- the kernels' launches -----------------------------------------------------------------------------
// Workgroups of a compute unit: what the registers allow (a fourth one where 16 rows of 128 channels leave room gains nothing; four column
// tiles of 128 channels: two 40 us, one 42, at 16 sequences of 3001, 8 kv heads and 64 rows).
constexpr int stream_groups(int d, int qt, int waves) { return waves == 8 ? 1 : d * qt <= 128 ? 3 : 2; }
void launch_stream(const AttentionArgs& a, int head_dim, int scale_group, int qt, int waves, unsigned grid, hipStream_t stream);  // 8 only up to D = 128, there for any qt, below for qt = 1
void launch_tile(const AttentionArgs& a, int head_dim, int scale_group, int waves, unsigned grid, hipStream_t stream);  // 8 only up to D = 128

}  // namespace ams_kv
#endif
