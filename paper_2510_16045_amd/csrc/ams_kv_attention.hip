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
// Split of the work: the host knows neither lengths nor (with row starts) how many rows a sequence has, so every workgroup works it
// out from them: the steps of all row tiles of a kv head, one tile after the other, are cut into equal shares, as many as there are
// workgroups that fit on the chip at once.  A share may begin and end inside a tile; that a workgroup begins a tile counts as much as
// kTileSteps steps.  Where no tile has more than kUncutSteps, shares are made of whole tiles.  Of a tile that lies in several shares every
// workgroup leaves its part (max, sum, O) in the workspace and counts itself in; the one that comes last adds all of them up, always in
// the same order, and clears the count.  Nobody waits for anybody.
#include "ams_kv.h"

#include <float.h>

#include <algorithm>

namespace ams_kv {

constexpr int kDeviceScope = 16;  // cache policy (sc1) of a buffer load or store that the whole device sees
constexpr int kStep = 32;         // keys of a wavefront's step
constexpr int kMinShare = 16;     // steps of a share: four for each wavefront
constexpr int kTileSteps = 14;    // what it takes to begin a tile and to leave its result, in steps
constexpr int kUncutSteps = 32;   // a tile of so many is not cut: joining its parts takes longer than its steps
constexpr int kMaxParts = 64;     // a tile in more parts costs its last workgroup more than the others gain
constexpr float kLift = 8.0f;     // exponents of P are raised by this: below it P keeps fp16's full precision over 2^-22 of the largest
constexpr float kSlack = 7.0f;    // how far (log2) a score may pass the running maximum before that is raised: 2^(8 + 7) is in fp16

struct AttentionArgs {
  View v;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  uint32_t* counts;  // [kv head][share in which the tile begins]
  float* parts;      // [kv head][2 share + (the tile begins in it)][row of the tile][max, sum, -, -, D values]
  int64_t q_stride, q_head, out_stride, out_head, lse_stride;
  float scale2;  // softmax_scale * log2(e)
  int group;     // R
  Divisor by_group;
  int shares;        // workgroups of one kv head
  int cut;           // whether a tile may lie in several
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

__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x += (uint32_t)__shfl_xor((int)x, i, 64);
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ int wave_prefix(int x) {  // inclusive
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int y = __shfl_up(x, i, 64);
    if (lane_id() >= i) x += y;
  }
  return x;
}
// x, of which the compiler knows nothing: what follows from it is not worked out before it is needed and kept in registers.
__device__ __forceinline__ int hidden(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int of_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// How much a share is, and all row tiles together: in steps with kTileSteps more for each tile, or in tiles that are not cut.
struct Split {
  uint32_t per, total;
  bool cut;
};
__device__ __forceinline__ uint32_t tile_cost(const Extent& e, bool cut) { return cut ? e.steps + kTileSteps : 1; }
template <int ROWS>
__device__ __forceinline__ Split split_of(const AttentionArgs& a, const Extent& first) {  // first: of the first 64 sequences
  uint32_t tiles = first.row_tiles, cost = first.row_tiles * tile_cost(first, true), most = first.row_tiles > 0 ? first.steps : 0;
  for (int b0 = 64; b0 < a.v.batch; b0 += 64) {
    const Extent x = extent_of<ROWS>(a, b0 + lane_id());
    tiles += x.row_tiles, cost += x.row_tiles * tile_cost(x, true), most = max(most, x.row_tiles > 0 ? (uint32_t)x.steps : 0);
  }
  Split split;
  split.cut = a.cut && __ballot(most > (uint32_t)kUncutSteps) != 0;
  split.total = wave_sum(split.cut ? cost : tiles);
  split.per = (split.total + a.shares - 1) / (uint32_t)a.shares;
  if (split.cut) split.per = max(split.per, (uint32_t)kMinShare);
  return split;
}

// The row tile that the cost `at` of the whole falls on, where its own begins and how much it is.
struct Place {
  Extent e;
  int b, row_tile;
  uint32_t first, cost;
};
template <int ROWS>
__device__ __forceinline__ bool place_of(const AttentionArgs& a, Extent e, bool cut, uint32_t at, Place* out) {  // e: of the first 64 sequences
  uint32_t before = 0;
  for (int b0 = 0; b0 < a.v.batch; b0 += 64) {
    if (b0 > 0) e = extent_of<ROWS>(a, b0 + lane_id());
    const uint32_t each = tile_cost(e, cut), mine = e.row_tiles * each;
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

// The pages of 64 steps of a wavefront, one step to a lane: looked up together, read lane by lane.
struct Pages {
  int number[2];  // of each tile of the step: -1 where the table names no page
  __device__ __forceinline__ void look_up(const AttentionArgs& a, int b, int step, int to) {
#pragma unroll
    for (int t = 0; t < 2; t++) {
      const uint32_t page = a.v.page_tiles.quotient((uint32_t)(2 * step + t));
      int found = -1;
      if (step < to && page < (uint32_t)a.v.table_width) found = a.v.table[b * a.v.table_stride + page];
      number[t] = (uint32_t)found < (uint32_t)a.v.n_pages ? found : -1;
    }
  }
};

// A tile's block as a buffer; of a page that is not there nothing is read.
struct Tile {
  __amdgpu_buffer_rsrc_t block;
  int tile;   // in its page
  bool held;  // there is a page
  __device__ __forceinline__ Tile(const AttentionArgs& a, const Pages& pages, int head, int step, int t, int at) {
    const int number = of_lane(pages.number[t], at);
    held = number >= 0;
    const uint64_t begin = (uint64_t)a.v.pages + (uint64_t)(held ? number : 0) * (uint64_t)a.v.page_bytes + (uint64_t)(uint32_t)head * (uint32_t)a.v.block;
    block = __builtin_amdgcn_make_buffer_rsrc((void*)begin, 0, held ? a.v.block : 0, 0x00020000);
    const uint32_t index = 2 * step + t;
    tile = (int)(index - a.v.page_tiles.quotient(index) * a.v.page_tiles.by);
  }
};

// A lane's words of the two tiles of a step and their scales.  V's scales are asked for once by the lanes together, 8 RUNS words of
// 32 bits of a tile.
template <int D, int G>
struct StepK {
  static constexpr int RUNS = D / G;
  Lane<D> w[2];
  Scales<RUNS> s[2];
  __device__ __forceinline__ void load(const AttentionArgs& a, const Tile& from, int t, uint32_t lane) {
    load_words<D>(w[t], from.block, lane, from.tile * 8 * D);
    s[t].load(from.block, (lane & 15) * (RUNS * 2u), 2 * a.v.codes + from.tile * kTile * RUNS * 2);
  }
};
template <int D, int G>
struct StepV {
  static constexpr int RUNS = D / G;
  Lane<D> w[2];
  uint32_t s[2];
  __device__ __forceinline__ void load(const AttentionArgs& a, const Tile& from, int t, uint32_t lane) {
    load_words<D>(w[t], from.block, lane, a.v.codes + from.tile * 8 * D);
    s[t] = __builtin_amdgcn_raw_buffer_load_b32(from.block, lane < 8 * RUNS ? lane * 4 : 0x7FFE0000, 2 * a.v.codes + a.v.scales + from.tile * kTile * RUNS * 2, 0);
  }
};

// Runs of V that stand for NaN take part in a step's products as zeros where not every row sees every key of the step, and the rows
// that do see one get the NaN here.  stage: the scales of the step's two tiles; begin, end: the keys that a lane's row sees.
template <int RUNS, int G, int QT, int DT>
__device__ __forceinline__ void nan_of_seen_keys(uint8_t* stage, int lane, int first_key, const int (&begin)[QT], const int (&end)[QT], f4 (&o)[DT][QT]) {
  const int g = lane >> 4;
  uint32_t bad[RUNS], any = 0;  // of the step's 32 keys those whose run stands for NaN; first a lane's eight
#pragma unroll
  for (int run = 0; run < RUNS; run++) {
    bad[run] = 0;
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++)
        if ((*(const uint16_t*)(stage + ((u * 4 + g) * RUNS + run) * 8 + 2 * j) & 0x7C00) == 0x7C00) bad[run] |= 1u << (16 * u + 4 * g + j);
    any |= bad[run];
  }
  if (!__ballot(any != 0)) return;
#pragma unroll
  for (int run = 0; run < RUNS; run++) {
    bad[run] |= (uint32_t)__shfl_xor((int)bad[run], 16, 64);
    bad[run] |= (uint32_t)__shfl_xor((int)bad[run], 32, 64);
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (bad[run] >> (16 * u + 4 * g + j) & 1) *(uint16_t*)(stage + ((u * 4 + g) * RUNS + run) * 8 + 2 * j) = 0;
#pragma unroll
    for (int t = 0; t < QT; t++) {
      const int from = min(max(begin[t] - first_key, 0), 32), to = min(max(end[t] - first_key, 0), 32);
      const uint32_t seen = (uint32_t)((1ull << to) - 1) & ~(uint32_t)((1ull << from) - 1);
      if (bad[run] & seen) {
#pragma unroll
        for (int d = run * G / 16; d < (run + 1) * G / 16; d++) o[d][t] = f4{NAN, NAN, NAN, NAN};
      }
    }
  }
  wave_sync();
}

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

// Adds up the parts of a row tile.  D / 4 lanes take a row, four channels each; of the workgroup's groups of
// lanes as many take the rows as there are (a power of two), and the others share the parts of a row; 8 parts are asked for before the
// first is used.
template <int D, int THREADS>
__device__ __forceinline__ void join_parts(const AttentionArgs& a, const Pending& tile, __amdgpu_buffer_rsrc_t left, int head, float* lds) {
  constexpr int LANES = D / 4, GROUPS = THREADS / LANES, AHEAD = 8;
  f4* const xs = (f4*)lds;             // [group][lane]
  f2* const stats = (f2*)(xs + THREADS);  // [group]
  const int group = threadIdx.x / LANES, c = threadIdx.x % LANES;
  const int rows = tile.rows, first = tile.first, count = tile.count;
  int takers = 1;  // groups that take rows
  while (takers < rows && takers < GROUPS) takers *= 2;
  const int sharers = GROUPS / takers, mine = group / takers;
  for (int i0 = 0; i0 < rows; i0 += takers) {
    const int i = i0 + group % takers;
    float top = -INFINITY, sum = 0;
    f4 x = {0, 0, 0, 0};
    for (int s0 = mine; s0 < count; s0 += sharers * AHEAD) {
      f4 from[AHEAD];
      f2 stat[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; j++) {
        const int s = s0 + j * sharers;
        const int at = s < count && i < rows ? ((2 * (first + s) + (s == 0)) * a.part_rows + i) * (D + 4) * 4 : 0x7FFE0000;  // nothing is read there
        from[j] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(left, at + 16 + 16 * c, 0, kDeviceScope));
        stat[j] = __builtin_bit_cast(f2, __builtin_amdgcn_raw_buffer_load_b64(left, at, 0, kDeviceScope));
        if (s >= count) stat[j] = f2{-INFINITY, 0};
      }
      float most = top;
#pragma unroll
      for (int j = 0; j < AHEAD; j++) most = fmaxf(most, stat[j][0]);
      const float less = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - most);
      top = most;
      sum *= less, x *= less;
#pragma unroll
      for (int j = 0; j < AHEAD; j++) {
        const float by = stat[j][0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(stat[j][0] - top);
        sum += stat[j][1] * by;
        x += from[j] * by;
      }
    }
    __syncthreads();  // what was in LDS has been read
    xs[threadIdx.x] = x;
    if (c == 0) stats[group] = f2{top, sum};
    __syncthreads();
    if (mine == 0 && i < rows) {
      top = -INFINITY, sum = 0;
      x = f4{0, 0, 0, 0};
      for (int j = 0; j < sharers; j++) top = fmaxf(top, stats[j * takers + group][0]);
      for (int j = 0; j < sharers; j++) {
        const f2 stat = stats[j * takers + group];
        const float by = stat[0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(stat[0] - top);
        sum += stat[1] * by;
        x += xs[(j * takers + group) * LANES + c] * by;
      }
      store_out(a, tile.start, head, tile.row0 + i, 4 * c, x * (sum > 0 || sum != sum ? 1.0f / sum : 0.0f));
      if (c == 0) store_lse(a, tile.start, head, tile.row0 + i, top, sum);
    }
  }
}

// Wavefronts of a workgroup, and workgroups of a compute unit: what the registers allow.
constexpr int stream_waves(int, int) { return 4; }
constexpr int stream_groups(int d, int qt) { return d * qt <= 128 ? 3 : d * qt < 512 ? 2 : 1; }

template <int D, int G, int QT>
__global__ __launch_bounds__(64 * stream_waves(D, QT), stream_groups(D, QT) * stream_waves(D, QT) / 4) void stream_kernel(AttentionArgs a) {
  constexpr int kStreamWaves = stream_waves(D, QT), ROWS = 16 * QT, RUNS = D / G, DT = D / 16, KB = D / 32, AT_ONCE = DT < 8 ? DT : 8;
  const int wave = uniform((int)threadIdx.x >> 6), lane = lane_id();
  const int share = (int)a.v.heads.quotient(blockIdx.x), head = blockIdx.x - share * a.v.kv_heads;
  // While keys are read: the rows of q as the matrix instructions take them, and V's scales of each wavefront's step.  Then the
  // wavefronts' results, eight d-tiles of a column tile at a time.
  constexpr int Q_BYTES = KB * QT * 1024, STAGE = 64 * RUNS, PARTS = kStreamWaves * AT_ONCE * 1024;
  __shared__ __align__(16) uint8_t shared[Q_BYTES + kStreamWaves * STAGE > PARTS ? Q_BYTES + kStreamWaves * STAGE : PARTS];
  __shared__ float tops[kStreamWaves][ROWS], sums[kStreamWaves][ROWS];
  __shared__ bool all_there[2];
  h8* const q_rows = (h8*)shared;
  uint8_t* const stage = shared + Q_BYTES + wave * STAGE;
  f4* const parts = (f4*)shared;

  const Extent first_64 = extent_of<ROWS>(a, lane);
  const Split split = split_of<ROWS>(a, first_64);
  uint32_t now = share * split.per;
  const uint32_t stop = min(now + split.per, split.total);
  const __amdgpu_buffer_rsrc_t left = __builtin_amdgcn_make_buffer_rsrc((void*)(a.parts + (int64_t)uniform(head) * 2 * a.shares * a.part_rows * (D + 4)), 0,
                                                                        a.cut ? 2 * a.shares * a.part_rows * (D + 4) * 4 : 0, 0x00020000);  // this head's parts
  Place place;
  Pending left_first = {}, left_last = {};
  int pending = 0;
  while (now < stop && place_of<ROWS>(a, first_64, split.cut, now, &place)) {
    const Extent& e = place.e;
    const int rows = e.n * a.group, row0 = place.row_tile * ROWS;
    // the share's steps of the tile that some row sees, and the keys that every row sees
    const uint32_t then = min(place.first + place.cost, stop);
    const int begin_step = split.cut ? max((int)(now - place.first) - kTileSteps, 0) : 0, end_step = split.cut ? (int)(then - place.first) - kTileSteps : e.steps;
    now = then;
    if (end_step <= 0) break;  // the tile begins in the next share
    const bool alone = begin_step == 0 && end_step == e.steps;
    const int last_row = min(row0 + ROWS, rows) - 1;
    const int p_first = e.len - e.n + (int)a.by_group.quotient((uint32_t)row0), p_last = e.len - e.n + (int)a.by_group.quotient((uint32_t)last_row);
    const int from = uniform(max(e.lo / kStep + begin_step, key_begin(a, p_first) / kStep));
    const int to = uniform(min(e.lo / kStep + end_step, (key_end(a, e.len, p_last) + kStep - 1) / kStep));
    const int whole_begin = uniform(key_begin(a, p_last)), whole_end = uniform(key_end(a, e.len, p_first));
    Pages pages;
    pages.look_up(a, place.b, from + wave + kStreamWaves * hidden(lane), to);
    // the tile's rows: a lane has one of each column tile
    const int load_lane = hidden(lane);
#pragma unroll
    for (int t = 0; t < QT; t++) {
      const int r = row0 + 16 * t + (load_lane & 15), token = (int)a.by_group.quotient((uint32_t)r);
      const uint16_t* src = a.q + (int64_t)(e.start + token) * a.q_stride + (int64_t)(head * a.group + r - token * a.group) * a.q_head + 8 * (load_lane >> 4);
#pragma unroll
      for (int i0 = 0; i0 < KB; i0 += kStreamWaves) {
        const int i = i0 + wave;
        if (KB < kStreamWaves && i >= KB) break;
        u4 x = {0, 0, 0, 0};
        if (r < rows) x = load_half8(src + 32 * i, a.vec);
        q_rows[(i * QT + t) * 64 + lane] = __builtin_bit_cast(h8, x);
      }
    }
    __syncthreads();

    f4 o[DT][QT];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; t++) {
      m[t] = -INFINITY, l[t] = 0;
#pragma unroll
      for (int d = 0; d < DT; d++) o[d][t] = f4{0, 0, 0, 0};
    }
    // S^T of the two tiles of a step: a lane has four keys of each and its row.
    auto scores = [&](const StepK<D, G>& k, f4(&s)[2][QT]) {
#pragma unroll
      for (int i = 0; i < KB; i++) {
        const h8 k0 = restore_k(k.w[0].w[i], k.s[0].twice(32 * i / G)), k1 = restore_k(k.w[1].w[i], k.s[1].twice(32 * i / G));
#pragma unroll
        for (int t = 0; t < QT; t++) {
          const h8 q = q_rows[(i * QT + t) * 64 + lane];
          s[0][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q, i ? s[0][t] : f4{0, 0, 0, 0}, 0, 0, 0);
          s[1][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q, i ? s[1][t] : f4{0, 0, 0, 0}, 0, 0, 0);
        }
      }
    };
    // P from S, and the statistics.  The maximum is raised only where a score passes it by more than the slack, then for all lanes that
    // share the row.
    auto weights = [&](f4(&s)[2][QT], h8(&p)[QT]) {
#pragma unroll
      for (int t = 0; t < QT; t++) {
        float top = s[0][t][0];
#pragma unroll
        for (int i = 1; i < 8; i++) top = fmaxf(top, s[i / 4][t][i % 4]);
        top *= a.scale2;
        if (__ballot(top > m[t] + kSlack)) {
          top = fmaxf(top, m[t]);
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
    };
    // O^T += V^T P^T; scale(tile, word): a word of the tile's scales, two tokens of a run
    auto multiply = [&](const StepV<D, G>& v, const h8(&p)[QT], auto scale) {
#pragma unroll
      for (int i = 0; i < KB; i++) {
        u2 va[2], vb[2];
#pragma unroll
        for (int u = 0; u < 2; u++) {
          const u2 s = scale(u, 32 * i / G);
          restore_v(v.w[u].w[i], s[0], s[1], &va[u], &vb[u]);
        }
#pragma unroll
        for (int t = 0; t < QT; t++) {
          o[2 * i][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join_halves(va[0], va[1]), p[t], o[2 * i][t], 0, 0, 0);
          o[2 * i + 1][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join_halves(vb[0], vb[1]), p[t], o[2 * i + 1][t], 0, 0, 0);
        }
      }
    };
    auto put_scales = [&](const StepV<D, G>& v) {
      wave_sync();  // the last step's have been read
#pragma unroll
      for (int u = 0; u < 2; u++)
        if (lane < 8 * RUNS) *(uint32_t*)(stage + 32 * RUNS * u + 4 * lane) = v.s[u];
      wave_sync();
    };
    // The next step's keys are asked for as soon as this one's have been used, and its values then; behind the last step that one's
    // again, so that what is waited for is always the older request.
    int step = from + wave, at = 0;
    if (step < to) {
      StepK<D, G> k;
      StepV<D, G> v;
#pragma unroll
      for (int u = 0; u < 2; u++) {
        const Tile tile(a, pages, head, step, u, 0);
        k.load(a, tile, u, lane), v.load(a, tile, u, lane);
      }
      for (;;) {
        f4 s[2][QT];
        h8 p[QT];
        scores(k, s);
        const bool held[2] = {of_lane(pages.number[0], at) >= 0, of_lane(pages.number[1], at) >= 0};
        const bool whole = step * kStep >= whole_begin && (step + 1) * kStep <= whole_end && held[0] && held[1];  // every row sees every key
        const bool more = step + kStreamWaves < to;
        if (more && ++at == 64) {
          at = 0;
          pages.look_up(a, place.b, step + kStreamWaves + kStreamWaves * hidden(lane), to);
        }
        const int next = more ? step + kStreamWaves : step;
        const Tile t0(a, pages, head, next, 0, at), t1(a, pages, head, next, 1, at);
        k.load(a, t0, 0, lane), k.load(a, t1, 1, lane);
        int begin[QT], end[QT];
        if (!whole) {
          const int mine = hidden(lane), key = step * kStep + 4 * (mine >> 4);
#pragma unroll
          for (int t = 0; t < QT; t++) {
            const int r = row0 + 16 * t + (mine & 15), position = e.len - e.n + (int)a.by_group.quotient((uint32_t)r);
            begin[t] = r < rows ? key_begin(a, position) : 0;
            end[t] = r < rows ? key_end(a, e.len, position) : 0;
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
              for (int i = 0; i < 4; i++)
                if (key + 16 * u + i < begin[t] || key + 16 * u + i >= end[t] || !held[u]) s[u][t][i] = -INFINITY;
          }
        }
        weights(s, p);
        put_scales(v);
        if (!whole) nan_of_seen_keys<RUNS, G, QT, DT>(stage, hidden(lane), step * kStep, begin, end, o);
        multiply(v, p, [&](int u, int run) { return *(const u2*)(stage + ((u * 4 + (lane >> 4)) * RUNS + run) * 8); });
        v.load(a, t0, 0, lane), v.load(a, t1, 1, lane);
        if (!more) break;
        step = next;
      }
    }

    // The wavefronts' results are joined in their order.
    const int done = hidden(lane), g = done >> 4, col = done & 15;
#pragma unroll
    for (int t = 0; t < QT; t++) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
      if (g == 0) tops[wave][16 * t + col] = m[t], sums[wave][16 * t + col] = l[t];
    }
    const int part = (2 * share + (begin_step == 0)) * a.part_rows;
#pragma unroll
    for (int t = 0; t < QT; t++) {
      const int r = row0 + 16 * t + col;
      float top = -INFINITY, sum = 0, by[kStreamWaves], scale = 0;
#pragma unroll
      for (int d0 = 0; d0 < DT; d0 += AT_ONCE) {
        __syncthreads();
#pragma unroll
        for (int d = 0; d < AT_ONCE; d++) parts[(wave * AT_ONCE + d) * 64 + done] = o[d0 + d][t];
        __syncthreads();
        if (d0 == 0) {
#pragma unroll
          for (int w = 0; w < kStreamWaves; w++) top = fmaxf(top, tops[w][16 * t + col]);
#pragma unroll
          for (int w = 0; w < kStreamWaves; w++) {
            const float mine = tops[w][16 * t + col];
            by[w] = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
            sum += sums[w][16 * t + col] * by[w];
          }
          scale = alone ? (sum > 0 || sum != sum ? 1.0f / sum : 0.0f) : 1.0f;
        }
        for (int d = wave; d < AT_ONCE; d += kStreamWaves) {
          f4 x = {0, 0, 0, 0};
#pragma unroll
          for (int w = 0; w < kStreamWaves; w++) x += parts[(w * AT_ONCE + d) * 64 + done] * by[w];
          if (r >= rows) continue;
          const int channel = 16 * (d0 + d) + 4 * g;
          if (alone)
            store_out(a, e.start, head, r, channel, x * scale);
          else
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x), left, ((part + 16 * t + col) * (D + 4) + 4 + channel) * 4, 0, kDeviceScope);
        }
      }
      if (wave == 0 && g == 0 && r < rows) {
        if (alone)
          store_lse(a, e.start, head, r, top, sum);
        else
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, f2{top, sum}), left, (part + 16 * t + col) * (D + 4) * 4, 0, kDeviceScope);
      }
    }
    if (!alone) {
      const int first = (int)((place.first + kTileSteps) / split.per), last = (int)((place.first + kTileSteps + e.steps - 1) / split.per);
      left_first = pending == 0 ? Pending{e.start, row0, min(rows - row0, ROWS), first, last - first + 1} : left_first;
      left_last = Pending{e.start, row0, min(rows - row0, ROWS), first, last - first + 1};
      pending++;
    }
    __syncthreads();  // what the tile left in LDS has been read
  }
  // Only the first and the last tile of a share may lie in others too.  Every wavefront's stores have been acknowledged before the
  // workgroup is counted in, and the parts are asked for after the count has come back; they go to the level of the memory system that
  // all compute units share.
  if (pending == 0) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x < (unsigned)pending) {
    const Pending mine = threadIdx.x == 0 ? left_first : left_last;
    uint32_t* const counter = a.counts + head * a.shares + mine.first;
    const bool last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)mine.count - 1;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all_there[threadIdx.x] = last;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i < pending; i++)
    if (all_there[i]) join_parts<D, 64 * kStreamWaves>(a, i == 0 ? left_first : left_last, left, head, (float*)shared);
}

// ---- launch ------------------------------------------------------------------------------------------
constexpr int kComputeUnits = 256;
constexpr size_t kCountBytes = 64 * 1024;  // of a workspace: counts of any call (kv_heads x shares of them), at its front
static_assert(4 * kComputeUnits * sizeof(uint32_t) <= kCountBytes && AMS_KV_MAX_HEADS * sizeof(uint32_t) <= kCountBytes, "one for each share of each head");

struct Plan {
  int qt, rows, part_rows;
  int64_t row_tiles;  // at most so many over all sequences
  int64_t shares;
  bool cut;
  size_t workspace;   // bytes that this many shares need
};
Plan make_plan(const ams_kv_cache* c, int64_t rows, int heads, int64_t max_q_len, size_t workspace) {
  Plan p;
  const int R = heads / c->kv_heads;
  const int64_t most = (c->q_starts ? std::min(max_q_len > 0 ? max_q_len : rows, rows) : 1) * R;
  p.qt = most <= 16 ? 1 : most <= 32 || c->head_dim == 256 ? 2 : 4;
  p.rows = 16 * p.qt;
  p.row_tiles = c->q_starts ? rows * R / p.rows + c->batch : c->batch * (int64_t)((R + p.rows - 1) / p.rows);
  const int64_t tile_steps = std::max<int64_t>(((int64_t)c->table_width * c->page_size + kStep - 1) / kStep, 1);
  p.part_rows = (int)std::min<int64_t>(c->q_starts ? rows * R : R, p.rows);
  const size_t part = (size_t)c->kv_heads * p.part_rows * (c->head_dim + 4) * sizeof(float);
  const size_t room = std::min<size_t>(workspace, AMS_KV_WORKSPACE_BYTES);
  const int64_t fit = std::max<int64_t>(stream_groups(c->head_dim, p.qt) * kComputeUnits / c->kv_heads, 1);
  p.shares = std::min(std::min(fit, p.row_tiles * kMaxParts), room < kCountBytes ? 0 : (int64_t)((room - kCountBytes) / part / 2));
  p.cut = p.shares > 1 && tile_steps > kUncutSteps && p.row_tiles * (tile_steps + kTileSteps) <= 0x7FFFFFFF;
  p.workspace = p.cut ? kCountBytes + 2 * (size_t)p.shares * part : 0;
  if (!p.cut) p.shares = p.row_tiles;
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
  a.q = Q, a.out = O, a.lse = lse, a.counts = (uint32_t*)workspace, a.parts = (float*)((uint8_t*)workspace + kCountBytes);
  a.q_stride = q_stride, a.q_head = q_head_stride, a.out_stride = o_stride, a.out_head = o_head_stride, a.lse_stride = lse_stride;
  a.scale2 = softmax_scale * 1.44269504089f;
  a.group = heads / cache->kv_heads, a.by_group = divisor((uint32_t)a.group);
  a.causal = causal != 0, a.window = (int)std::min<int64_t>(window, 0x3FFFFFFF);
  a.vec = aligned(Q, 16) && aligned(O, 8) && (q_stride | q_head_stride) % 8 == 0 && (o_stride | o_head_stride) % 4 == 0;
  const Plan p = make_plan(cache, rows, heads, max_q_len, workspace ? workspace_bytes : 0);
  a.shares = (int)p.shares, a.cut = p.cut, a.part_rows = p.part_rows;
  const int64_t grid = p.shares * cache->kv_heads;
  if (grid > 0x7FFFFFFF) return AMS_ERR_SHAPE;
  dispatch(cache->head_dim, cache->scale_group, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    auto launch = [&](auto kernel, int qt) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * stream_waves(D, qt)), 0, (hipStream_t)stream, a); };
    switch (p.qt) {
      case 1: launch(stream_kernel<D, G, 1>, 1); break;
      case 2: launch(stream_kernel<D, G, 2>, 2); break;
      default:
        if constexpr (D < 256) launch(stream_kernel<D, G, 4>, 4);  // 256 accumulators do not fit beside the rows
    }
  });
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

}  // extern "C"
