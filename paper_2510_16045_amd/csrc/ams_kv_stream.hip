// Attention over the 4-bit KV cache for few rows of a kv head (single tokens, drafts), and for more of them where keys have to be shared
// out to fill the chip.
//
// stream_kernel: one read of the cache.  A workgroup takes a tile of 16 QT rows and a share of the keys; its wavefronts take turns at steps
// of 32 keys, straight from memory to registers: K's words become the A operand of S^T = K q^T, the result lies as the B operand of
// O^T = V^T P^T wants it (a lane has the same four keys of a tile in both), and V's words become its A operand, so that neither the cache
// nor P passes through LDS.  LDS holds what all lanes need: the rows of q, the scales of a wavefront's step of V, at the end the
// wavefronts' sums.  The running maximum is the wavefront's own until then.
//
// What bounds it is memory and the way to it.  32 sequences of 819 to 8192 tokens, 32 query and 8 kv heads of 128 channels, runs of 32:
// 165 MB in 41 us, 4.0 TB/s; one sequence of 131071, runs of 64: 143 MB in 36.5 us.  A bare read of these bytes takes 23 and 20 us, and
// the loop comes near that (21 to 26); 5 us pass before the first keys are there (lengths, table, cache: three trips, each from the
// last one's answer), 5 to 8 at the end (parts out, count, parts in).  The vector units are busy for 16 of the 40 us (280
// instructions a step of 32 keys and 16 rows, 112 of them the conversion of codes and their scaling), the matrix units for 4.  Five rows of
// 16 sequences of 3001 tokens, 64 and 8 heads, tiles of 40 rows: 57 MB in 27 us; 560 instructions a step, 11 us of them.
#include "ams_kv_attention.h"

namespace ams_kv {

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
// 32 bits of a tile, and handed round through LDS: a lane needs those of its four keys in all runs, which takes RUNS loads of its own.
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
// that do see one get the NaN here.  So do runs whose scale is none that ams_kv_write stores (bits above kTopScale): they lie where no row has been
// written, where a pool may hold anything, and a value that is no fp16 value any more would turn the 0 of a key that is not seen into a
// NaN as well.  stage: the scales of the step's two tiles; begin, end: the keys that a lane's row sees.
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
        if (*(const uint16_t*)(stage + ((u * 4 + g) * RUNS + run) * 8 + 2 * j) > kTopScale) bad[run] |= 1u << (16 * u + 4 * g + j);
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

template <int D, int G, int QT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, stream_groups(D, QT, WAVES) * WAVES / 4) void stream_kernel(AttentionArgs a) {
  constexpr int ROWS = 16 * QT, RUNS = D / G, DT = D / 16, KB = D / 32, AT_ONCE = DT < 8 ? DT : 8;
  const int wave = uniform((int)threadIdx.x >> 6), lane = lane_id();
  const int share = (int)a.v.heads.quotient(blockIdx.x), head = blockIdx.x - share * a.v.kv_heads;
  // While keys are read: the rows of q as the matrix instructions take them, and V's scales of each wavefront's step.  Then the
  // wavefronts' results, eight d-tiles of a column tile at a time.
  constexpr int Q_BYTES = KB * QT * 1024, STAGE = 64 * RUNS, PARTS = WAVES * AT_ONCE * 1024;
  __shared__ __align__(16) uint8_t shared[Q_BYTES + WAVES * STAGE > PARTS ? Q_BYTES + WAVES * STAGE : PARTS];
  __shared__ float tops[WAVES][ROWS], sums[WAVES][ROWS];
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
  while (now < stop && place_of<ROWS>(a, first_64, split, now, &place)) {
    const Extent& e = place.e;
    const int rows = e.n * a.group, row0 = place.row_tile * ROWS;
    // the share's steps of the tile that some row sees, and the keys that every row sees
    const uint32_t then = min(place.first + place.cost, stop);
    int begin_step = 0, end_step = e.steps;
    if (split.cut && split.pieces > 0) {
      const uint32_t part = now - place.first;
      const float each = (float)e.steps * __builtin_amdgcn_rcpf((float)place.cost);
      begin_step = uniform((int)((float)part * each));
      end_step = part + 1 == place.cost ? e.steps : uniform((int)((float)(part + 1) * each));
    } else if (split.cut) {
      begin_step = max((int)(now - place.first) - kTileSteps, 0), end_step = (int)(then - place.first) - kTileSteps;
    }
    if (end_step <= 0 || then <= now) break;  // the tile begins in the next share (and starts that are not ascending end somewhere)
    now = then;
    const bool alone = begin_step == 0 && end_step == e.steps;
    const int last_row = min(row0 + ROWS, rows) - 1;
    const int p_first = e.len - e.n + (int)a.by_group.quotient((uint32_t)row0), p_last = e.len - e.n + (int)a.by_group.quotient((uint32_t)last_row);
    const int from = uniform(max(e.lo / kStep + begin_step, key_begin(a, p_first) / kStep));
    const int to = uniform(min(e.lo / kStep + end_step, (key_end(a, e.len, p_last) + kStep - 1) / kStep));
    const int whole_begin = uniform(key_begin(a, p_last)), whole_end = uniform(key_end(a, e.len, p_first));
    Pages pages;
    pages.look_up(a, place.b, from + wave + WAVES * hidden(lane), to);
    // the tile's rows: a lane has one of each column tile
    const int load_lane = hidden(lane);
#pragma unroll
    for (int t = 0; t < QT; t++) {
      const int r = row0 + 16 * t + (load_lane & 15), token = (int)a.by_group.quotient((uint32_t)r);
      const uint16_t* src = a.q + (int64_t)(e.start + token) * a.q_stride + (int64_t)(head * a.group + r - token * a.group) * a.q_head + 8 * (load_lane >> 4);
#pragma unroll
      for (int i0 = 0; i0 < KB; i0 += WAVES) {
        const int i = i0 + wave;
        if (KB < WAVES && i >= KB) break;
        u4 x = {0, 0, 0, 0};
        if (r < rows) x = load_half8(src + 32 * i, a.vec);
        q_rows[(i * QT + t) * 64 + lane] = __builtin_bit_cast(h8, x);
      }
    }
    __syncthreads();

    f4 o[DT][QT];
    float m[QT], l[QT];
    bool far = false;  // some row's maximum is beyond kFar
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
        if (__ballot(top - m[t] > kSlack)) {
          top = fmaxf(top, m[t]);
          top = larger(with_32(larger(with_16(top))));
          const float less = top > m[t] ? __builtin_amdgcn_exp2f(m[t] - top) : 1.0f;
          m[t] = top;
          far |= any_far(top);
          l[t] *= less;
#pragma unroll
          for (int d = 0; d < DT; d++) o[d][t] *= less;
        }
        float scale2 = a.scale2, sub = m[t] == -INFINITY ? 0.0f : m[t] - kLift;
        if (far) {
#pragma unroll
          for (int i = 0; i < 8; i++) s[i / 4][t][i % 4] = below_top(s[i / 4][t][i % 4], a.scale2, m[t]);
          scale2 = 1.0f, sub = -kLift;
        }
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][t][i], scale2, -sub));
            l[t] += v;
            p[t][4 * u + i] = (_Float16)v;  // as the matrix cores take it; 1.4e-4 to 2.9e-4 from 64 bits, with fp32 weights 1.4e-4 to 2.1e-4
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
        const bool more = step + WAVES < to;
        if (more && ++at == 64) {
          at = 0;
          pages.look_up(a, place.b, step + WAVES + WAVES * hidden(lane), to);
        }
        const int next = more ? step + WAVES : step;
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
      l[t] = sum_of(with_32(sum_of(with_16(l[t]))));
      if (g == 0) tops[wave][16 * t + col] = m[t], sums[wave][16 * t + col] = l[t];
    }
    const int part = (2 * share + (begin_step == 0)) * a.part_rows;
#pragma unroll
    for (int t = 0; t < QT; t++) {
      const int r = row0 + 16 * t + col;
      float top = -INFINITY, sum = 0, by[WAVES], scale = 0;
#pragma unroll
      for (int d0 = 0; d0 < DT; d0 += AT_ONCE) {
        __syncthreads();
#pragma unroll
        for (int d = 0; d < AT_ONCE; d++) parts[(wave * AT_ONCE + d) * 64 + done] = o[d0 + d][t];
        __syncthreads();
        if (d0 == 0) {
#pragma unroll
          for (int w = 0; w < WAVES; w++) top = fmaxf(top, tops[w][16 * t + col]);
#pragma unroll
          for (int w = 0; w < WAVES; w++) {
            const float mine = tops[w][16 * t + col];
            by[w] = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
            sum += sums[w][16 * t + col] * by[w];
          }
          scale = alone ? (sum > 0 || sum != sum ? 1.0f / sum : 0.0f) : 1.0f;
        }
        for (int d = wave; d < AT_ONCE; d += WAVES) {
          f4 x = {0, 0, 0, 0};
#pragma unroll
          for (int w = 0; w < WAVES; w++) x += parts[(w * AT_ONCE + d) * 64 + done] * by[w];
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
      const int first = split.pieces > 0 ? (int)place.first : min((int)((place.first + kTileSteps) / split.per), a.shares - 1);
      const int last = split.pieces > 0 ? (int)(place.first + place.cost) - 1 : (int)((place.first + kTileSteps + e.steps - 1) / split.per);
      left_first = pending == 0 ? Pending{e.start, row0, min(rows - row0, ROWS), first, last - first + 1} : left_first;
      left_last = Pending{e.start, row0, min(rows - row0, ROWS), first, last - first + 1};
      pending++;
    }
    __syncthreads();  // what the tile left in LDS has been read
  }
  join_pending<D, 64 * WAVES, QT == 1 ? 1 : 4, QT == 1 ? 8 : 4>(a, pending, left_first, left_last, left, share, head, (float*)shared, all_there);
}

bool load_stream() { return loaded((const void*)stream_kernel<64, 32, 1, 4>); }

void launch_stream(const AttentionArgs& a, int head_dim, int scale_group, int qt, int waves, unsigned grid, hipStream_t stream) {
  dispatch(head_dim, scale_group, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * waves), 0, stream, a); };
    if constexpr (D == 128) {
      if (waves == 8 && qt == 2) return launch(stream_kernel<D, G, 2, 8>);
      if (waves == 8 && qt == 3) return launch(stream_kernel<D, G, 3, 8>);
      if (waves == 8 && qt == 4) return launch(stream_kernel<D, G, 4, 8>);
    }
    if constexpr (D < 256) {
      if (waves == 8 && qt == 1) return launch(stream_kernel<D, G, 1, 8>);
      if (qt == 3) return launch(stream_kernel<D, G, 3, 4>);
      if (qt == 4) return launch(stream_kernel<D, G, 4, 4>);  // 256 accumulators do not fit beside the rows
    }
    if (qt == 1) return launch(stream_kernel<D, G, 1, 4>);
    launch(stream_kernel<D, G, 2, 4>);
  });
}

}  // namespace ams_kv
