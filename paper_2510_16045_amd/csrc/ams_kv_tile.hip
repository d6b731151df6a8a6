// Attention over the 4-bit KV cache for many rows: prompts.
//
// tile_kernel: a workgroup takes 32 rows for each of its wavefronts and walks the keys in blocks of 64.  A block is restored to fp16 once,
// by all wavefronts together (a tile of K or V each), into LDS in the order in which 32x32x16 matrix instructions take it, so that
// every read is 64 lanes of 16 bytes side by side; two blocks take turns, and the next but one is already on its way from memory.
// S^T = K q^T lies in registers as the B operand of O^T = V^T P^T wants it: a lane's keys of a 16-key tile are 4 h .. + 3 and
// 8 + 4 h .. + 3 (h = lane / 32), and V's fragments are laid out in that order.
//
// What bounds it is the issue of instructions, which two wavefronts of a SIMD share: 2048 rows over 8192 keys, 32 query and 8 kv heads of 128
// channels: 241 Gflop in 261 to 270 us, 0.89 to 0.92 Pflop/s, where a library product of 8192 x 8192 x 8192 reaches 1.16.  In copies with parts taken out:
// without restoring 235 us, without S too 165, without O too 136, without the softmax as well 101.  Tiles are never cut: keys of cut
// tiles were joined through the workspace at 340 us.  With a window of 512, seven sequences of up to 1999 tokens, 16 heads of 64: 41 us.
#include "ams_kv_attention.h"

namespace ams_kv {

typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kBlock = 64;                // keys
constexpr int kBlockTiles = kBlock / kTile;
// Fragments that are read ahead (2048 rows over 8192 keys of 128 channels: 2 269 us, 4 267, 8 271), and wavefronts of a SIMD: with 64 channels
// and workgroups of four there are registers for four, and two fragments (seven prompts of up to 1999, a window of 512, 16 heads:
// 49.9 -> 45.1 us; 16 of 2000 149 -> 142; 4 of 1024 over all keys 34.5 -> 35.5).
constexpr int ahead(int d, int waves) { return d == 64 && waves == 4 ? 2 : 4; }
constexpr int tile_waves(int d, int waves) { return d == 256 ? 1 : d == 64 && waves == 4 ? 4 : 2; }
constexpr int kReads = 0x100, kProducts = 0x008;  // of a scheduling group: LDS reads, matrix instructions

// What LDS holds of a block.
template <int D>
struct Block {
  h8 k[2][D / 16][64];            // [32 keys][16 channels][lane]
  h8 v[D / 32][kBlockTiles][64];  // [32 channels][16 keys][lane]
};
// Of its tiles: whether the table names no page, and whether V stands for NaN somewhere or has a scale that ams_kv_write does not
// store (bits above kTopScale), as there may be where no row has been written; if so the keys (bits), by run.
constexpr uint32_t kMissing = 1, kBad = 2;
template <int RUNS>
struct Notes {
  alignas(16) uint32_t what[kBlockTiles];  // read as one
  uint32_t bad[kBlockTiles][RUNS];
};
static_assert(alignof(Notes<1>) >= alignof(u4) && kBlockTiles == 4, "one read of 16 bytes");

// A tile of K or V on its way through a wavefront.
template <int D, int G>
struct Job {
  static constexpr int RUNS = D / G;
  uint32_t w[D / 32], s[2 * RUNS];
  bool held;
  __device__ __forceinline__ void load(const AttentionArgs& a, int number, int head, int tile, bool is_v, uint32_t lane) {
    held = number >= 0;
    const uint64_t begin = (uint64_t)a.v.pages + (uint64_t)(held ? number : 0) * (uint64_t)a.v.page_bytes + (uint64_t)(uint32_t)head * (uint32_t)a.v.block;
    const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)begin, 0, held ? a.v.block : 0, 0x00020000);  // of no page nothing is read
    const int in_page = (int)((uint32_t)tile - a.v.page_tiles.quotient((uint32_t)tile) * a.v.page_tiles.by);
    Lane<D> words;
    load_words<D>(words, from, lane, (is_v ? a.v.codes : 0) + in_page * 8 * D);
#pragma unroll
    for (int i = 0; i < D / 32; i++) w[i] = words.w[i];
    // both kinds by the same loads: a token's RUNS scales of K, which begin in the first word, or the 4 RUNS of four tokens of V
    const uint32_t mine = is_v ? (lane >> 4) * (RUNS * 8u) : (lane & 15) * (RUNS * 2u) & ~3u;
    const int scales = 2 * a.v.codes + (is_v ? a.v.scales : 0) + in_page * kTile * RUNS * 2;
    if constexpr (RUNS == 1) {
      const u2 x = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(from, mine, scales, 0));
      s[0] = x[0], s[1] = x[1];
    } else {
#pragma unroll
      for (int i = 0; i < 2 * RUNS; i += 4) {
        const u4 x = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(from, i == 0 || is_v ? mine + 4 * i : 0x7FFE0000u, scales, 0));
        s[i] = x[0], s[i + 1] = x[1], s[i + 2] = x[2], s[i + 3] = x[3];
      }
    }
  }
  __device__ __forceinline__ void store_k(Block<D>& block, int tile, int lane) const {
    const int g = lane >> 4, r = lane & 15;
    Scales<RUNS> x;
#pragma unroll
    for (int i = 0; i < Scales<RUNS>::WORDS; i++) x.w[i] = RUNS == 1 ? s[i] >> 16 * (r & 1) : s[i];
    h8* const to = &block.k[tile >> 1][g >> 1][(g & 1) * 32 + (tile & 1) * 16 + r];
#pragma unroll
    for (int i = 0; i < D / 32; i++) to[2 * i * 64] = restore_k(w[i], x.twice(32 * i / G));
  }
  __device__ __forceinline__ void store_v(Block<D>& block, Notes<RUNS>& notes, int tile, int lane) {
    const int q = lane >> 4, c = lane & 15;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 2 * RUNS; i++) most = max_halves(most, s[i]);
    const bool bad = (most & 0xFFFFu) > kTopScale || most >> 16 > kTopScale;
    const bool any = __ballot(bad) != 0;
    if (any) note_bad(notes, tile, lane);
    if (lane == 0) notes.what[tile] = (held ? 0 : kMissing) | (any ? kBad : 0);
    u2* const to = (u2*)&block.v[0][tile][(q & 1) * 32 + c] + (q >> 1);
#pragma unroll
    for (int i = 0; i < D / 32; i++) {
      u2 x, y;
      restore_v(w[i], s[32 * i / G * 2], s[32 * i / G * 2 + 1], &x, &y);
      to[i * kBlockTiles * 128] = x;
      to[i * kBlockTiles * 128 + 32] = y;
    }
  }
  // Such runs of V take part as zeros: what masks a key cannot be told from its 0 weight.  The rows that see one get the NaN.
  __device__ __forceinline__ void note_bad(Notes<RUNS>& notes, int tile, int lane) {
    const int q = lane >> 4;
#pragma unroll
    for (int run = 0; run < RUNS; run++) {
      uint32_t keys = 0;
#pragma unroll
      for (int j = 0; j < 4; j++)
        if ((s[2 * run + j / 2] >> 16 * (j & 1) & 0xFFFF) > kTopScale) {
          keys |= 1u << (4 * q + j);
          s[2 * run + j / 2] &= j & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
      keys |= (uint32_t)__shfl_xor((int)keys, 16, 64);
      keys |= (uint32_t)__shfl_xor((int)keys, 32, 64);
      if (lane == 0) notes.bad[tile][run] = keys;
    }
  }
};

template <int D, int G, int WAVES>
__global__ __launch_bounds__(64 * WAVES, tile_waves(D, WAVES)) void tile_kernel(AttentionArgs a) {
  constexpr int ROWS = 32 * WAVES, RUNS = D / G, KF = D / 16, DT = D / 32, JOBS = 2 * kBlockTiles / WAVES, AHEAD = ahead(D, WAVES);
  const int wave = uniform((int)threadIdx.x >> 6), lane = lane_id(), h = lane >> 5, col = lane & 31;
  const int share = (int)a.v.heads.quotient(blockIdx.x), head = blockIdx.x - share * a.v.kv_heads;
  __shared__ Block<D> blocks[2];
  __shared__ Notes<RUNS> notes[2];
  const Extent first_64 = extent_of<ROWS>(a, lane);
  const Split split = split_of<ROWS>(a, first_64);  // a tile each
  Place place;
  // the tiles with the most keys are a sequence's last: they go first
  if ((uint32_t)share < split.total && place_of<ROWS>(a, first_64, split, split.total - 1 - share, &place)) {
    const Extent& e = place.e;
    const int rows = e.n * a.group, tile_row = place.row_tile * ROWS, row0 = tile_row + 32 * wave;
    auto position = [&](int r) { return e.len - e.n + (int)a.by_group.quotient((uint32_t)r); };
    // the keys that some row of the tile sees, from a cache tile on
    const int key_from = uniform(key_begin(a, position(tile_row)) & ~(kTile - 1));
    const int key_to = uniform(key_end(a, e.len, position(min(tile_row + ROWS, rows) - 1)));
    const int n_blocks = max((key_to - key_from + kBlock - 1) / kBlock, 0);
    // of those the ones that every row and that no row of the wavefront sees
    const bool idle = row0 >= rows;
    const int p_first = position(row0), p_last = position(min(row0 + 32, rows) - 1);
    const int whole_begin = uniform(key_begin(a, p_last)), whole_end = uniform(min(key_end(a, e.len, p_first), key_to));
    const int some_begin = uniform(key_begin(a, p_first)), some_end = uniform(idle ? 0 : min(key_end(a, e.len, p_last), key_to));
    const int r = row0 + col;
    const int row_begin = key_begin(a, position(r)), row_end = r < rows ? min(key_end(a, e.len, position(r)), key_to) : 0;

    h8 q[KF];
    {
      const int token = (int)a.by_group.quotient((uint32_t)r);
      const uint16_t* const src = a.q + (int64_t)(e.start + token) * a.q_stride + (int64_t)(head * a.group + r - token * a.group) * a.q_head + 8 * h;
#pragma unroll
      for (int i = 0; i < KF; i++) {
        u4 x = {0, 0, 0, 0};
        if (r < rows) x = load_half8(src + 16 * i, a.vec);
        q[i] = __builtin_bit_cast(h8, x);
      }
    }
    f16v o[DT];
    float m = -INFINITY, l = 0;
    bool far = false;  // some row's maximum is beyond kFar
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int i = 0; i < 16; i++) o[d][i] = 0;

    // A wavefront's jobs: tile `wave % 4` of each block, of K, of V, or of both.
    const int my_tile = wave % kBlockTiles;
    int number = -1;  // the page of that tile in 64 blocks, one to a lane
    auto look_up = [&](int block) {
      const int tile = key_from / kTile + (block + hidden(lane)) * kBlockTiles + my_tile;
      const uint32_t page = a.v.page_tiles.quotient((uint32_t)tile);
      number = -1;
      if (tile * kTile < key_to && page < (uint32_t)a.v.table_width) {
        const int found = a.v.table[place.b * a.v.table_stride + page];
        if ((uint32_t)found < (uint32_t)a.v.n_pages) number = found;
      }
    };
    Job<D, G> jobs[JOBS];
    auto request = [&](int block) {
      if (block % 64 == 0) look_up(block);
#pragma unroll
      for (int j = 0; j < JOBS; j++)
        jobs[j].load(a, of_lane(number, block % 64), head, key_from / kTile + block * kBlockTiles + my_tile, JOBS == 1 ? wave >= kBlockTiles : j == 1, lane);
    };
    auto restore = [&](int buffer) {
#pragma unroll
      for (int j = 0; j < JOBS; j++) {
        if (JOBS == 1 ? wave >= kBlockTiles : j == 1)
          jobs[j].store_v(blocks[buffer], notes[buffer], my_tile, hidden(lane));
        else
          jobs[j].store_k(blocks[buffer], my_tile, hidden(lane));
      }
    };
    auto compute = [&](int buffer, int key0) {
      const Block<D>& block = blocks[buffer];
      // Fragments are read AHEAD instructions ahead of the one that takes them; left to itself the compiler reads each one where it is used
      // and waits for it.
      constexpr int NK = 2 * KF, NV = kBlockTiles * DT;
      const u4 what = *(const u4*)notes[buffer].what;
      h8 f[AHEAD];
      f16v s[2];
#pragma unroll
      for (int i = 0; i < 16; i++) s[0][i] = s[1][i] = 0;
#pragma unroll
      for (int n = 0; n < AHEAD; n++) f[n] = block.k[n & 1][n >> 1][lane];
#pragma unroll
      for (int n = 0; n < NK; n++) {
        s[n & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[n % AHEAD], q[n >> 1], s[n & 1], 0, 0, 0);
        if (n + AHEAD < NK) f[n % AHEAD] = block.k[(n + AHEAD) & 1][(n + AHEAD) >> 1][lane];
      }
      __builtin_amdgcn_sched_group_barrier(kReads, AHEAD, 0);
#pragma unroll
      for (int n = 0; n < NK; n++) {
        __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
        if (n + AHEAD < NK) __builtin_amdgcn_sched_group_barrier(kReads, 1, 0);
      }
#pragma unroll
      for (int n = 0; n < AHEAD; n++) f[n] = block.v[n % DT][n / DT][lane];
      const uint32_t anything = (uint32_t)uniform((int)(what[0] | what[1] | what[2] | what[3]));
      if (key0 < whole_begin || key0 + kBlock > whole_end || (anything & kMissing)) {  // some row does not see some key
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
          for (int i = 0; i < 16; i++) {
            const int key = key0 + 32 * kt + 8 * (i / 4) + 4 * h + i % 4;
            if (key < row_begin || key >= row_end || (what[2 * kt + i / 8] & kMissing)) s[kt][i] = -INFINITY;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 32; i++) top = fmaxf(top, s[i / 16][i % 16]);
      top *= a.scale2;
      float scale2 = a.scale2;
      if (far || __ballot(top - m > kSlack)) {  // the maximum is raised only where a score passes it by more than the slack
        top = fmaxf(top, m);
        top = larger(with_32(top));
        const float less = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
        m = top;
        far |= any_far(top);
        l *= less;
#pragma unroll
        for (int d = 0; d < DT; d++) o[d] *= less;
        if (far) {
#pragma unroll
          for (int i = 0; i < 32; i++) s[i / 16][i % 16] = below_top(s[i / 16][i % 16], a.scale2, top);
          scale2 = 1.0f;
        }
      }
      const float sub = far ? -kLift : m == -INFINITY ? 0.0f : m - kLift;
      h8 p[kBlockTiles];
      float sum[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 32; i++) {
        const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 16][i % 16], scale2, -sub));
        sum[i & 1] += v;
        p[i / 8][i % 8] = (_Float16)v;  // as in stream_kernel
      }
      l += sum[0] + sum[1];
#pragma unroll
      for (int n = 0; n < NV; n++) {
        o[n % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[n % AHEAD], p[n / DT], o[n % DT], 0, 0, 0);
        if (n + AHEAD < NV) f[n % AHEAD] = block.v[(n + AHEAD) % DT][(n + AHEAD) / DT][lane];
      }
#pragma unroll
      for (int n = 0; n < NV; n++) {
        __builtin_amdgcn_sched_group_barrier(kProducts, 1, 1);
        if (n + AHEAD < NV) __builtin_amdgcn_sched_group_barrier(kReads, 1, 1);
      }
      if (anything & kBad) {
#pragma unroll
        for (int run = 0; run < RUNS; run++) {
          bool seen = false;
          for (int t = 0; t < kBlockTiles; t++) {
            const int first = key0 + kTile * t, from = min(max(row_begin - first, 0), kTile), to = min(max(row_end - first, 0), kTile);
            if (what[t] & kBad) seen |= (notes[buffer].bad[t][run] & ((1u << to) - 1) & ~((1u << from) - 1)) != 0;
          }
          if (seen) {
#pragma unroll
            for (int d = run * G / 32; d < (run + 1) * G / 32; d++)
#pragma unroll
              for (int i = 0; i < 16; i++) o[d][i] = NAN;
          }
        }
      }
    };

    if (n_blocks > 0) {
      request(0);
      restore(0);
      if (n_blocks > 1) request(1);
      __syncthreads();
#pragma unroll 1
      for (int block = 0; block < n_blocks; block++) {
        if (block + 1 < n_blocks) restore((block + 1) & 1);
        if (block + 2 < n_blocks) request(block + 2);
        const int key0 = key_from + block * kBlock;
        if (key0 < some_end && key0 + kBlock > some_begin) compute(block & 1, key0);
        __syncthreads();
      }
    }

    l = sum_of(with_32(l));
    if (r < rows) {
      const float scale = l > 0 || l != l ? 1.0f / l : 0.0f;
#pragma unroll
      for (int d = 0; d < DT; d++)
#pragma unroll
        for (int i = 0; i < 16; i += 4) store_out(a, e.start, head, r, 32 * d + 2 * i + 4 * h, f4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]} * scale);
      if (h == 0) store_lse(a, e.start, head, r, m, l);
    }
  }
}

bool load_tile() { return loaded((const void*)tile_kernel<64, 32, 4>); }

void launch_tile(const AttentionArgs& a, int head_dim, int scale_group, int waves, unsigned grid, hipStream_t stream) {
  dispatch(head_dim, scale_group, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    if constexpr (D < 256) {
      if (waves == 8) {
        hipLaunchKernelGGL((tile_kernel<D, G, 8>), dim3(grid), dim3(512), 0, stream, a);
        return;
      }
    }
    hipLaunchKernelGGL((tile_kernel<D, G, 4>), dim3(grid), dim3(256), 0, stream, a);
  });
}

}  // namespace ams_kv
