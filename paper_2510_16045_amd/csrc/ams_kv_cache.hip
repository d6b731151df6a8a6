// Writing rows into the 4-bit KV cache and reading them back.
//
// Both are one pass over the rows: 4 D bytes of K and V per token and head on one side, D + 4 D / scale_group on the other.
// A wavefront takes a tile of 16 tokens of one head; the rows of a sequence are its last ones, so a tile is found from the row
// starts alone: sequence b has at most floor(rows / 16) + 2 tiles, and those of b begin at floor(start / 16) + 2 b.
//
// Memory bounds them, and the launch where there are few rows.  16384 rows of 8 heads of 128 channels, runs of 32: written in 19.8 us (86 MB,
// 4.3 TB/s), read back in 14.2 (6.1 TB/s; a copy of 1 GiB goes at 5.1, a bare read at 7.1); 131072 rows read back in 114 to 123 (5.6 to 6.0); one row for
// each of 32 sequences 4.5 and 3.3 us, where an empty launch takes 2.
#include "ams_kv.h"

namespace ams_kv {

// The rows of a wavefront's tile: rows `row` + r for r in [first, end), at position 16 tile + r (negative ones have no place).
struct TileRows {
  int b, tile, row, first, end;
};
__device__ __forceinline__ bool tile_rows(const View& v, int item, TileRows* t) {
  auto first_item = [&](int b) { return v.starts ? row_start(v, b) / kTile + 2 * b : b; };
  const int b = v.starts ? sequence_of(v.batch, item, first_item) : min(item, v.batch - 1);
  const int start = row_start(v, b), n = max(row_start(v, b + 1) - start, 0), len = kv_len(v, b);
  const int p0 = len - n;  // position of the first row
  const int tile = (p0 >> 4) + item - first_item(b);
  t->b = b, t->tile = tile, t->row = start + tile * kTile - p0;
  t->first = max(p0 - tile * kTile, 0), t->end = min(len - tile * kTile, kTile);
  return t->first < t->end;
}

// Eight halfs; rows that are not 16-byte aligned half by half.  They are read once, and stay out of the caches (16384 rows of 8 heads
// written and read back 45 -> 36 us).
__device__ __forceinline__ u4 load8(const uint16_t* p, bool vec) {
  if (vec) return __builtin_nontemporal_load((const u4*)p);
  u4 x;
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  return x;
}
__device__ __forceinline__ void store8(uint16_t* p, u4 x, bool vec) {
  if (vec) {
    __builtin_nontemporal_store(x, (u4*)p);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; i++) p[2 * i] = (uint16_t)x[i], p[2 * i + 1] = (uint16_t)(x[i] >> 16);
}

// A lane's value from another lane of its 16, by a data-parallel pattern.
template <int PATTERN>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, PATTERN, 0xF, 0xF, true);
}
constexpr int kSwapOne = 0xB1, kSwapTwo = 0x4E, kMirrorEight = 0x141, kMirror = 0x140;  // lane ^ 1, lane ^ 2, 7 - lane, 15 - lane

// The larger of a lane's value and those of the lanes that hold the rest of its run (4, 8 or 16 neighbours).
template <int LANES>
__device__ __forceinline__ uint32_t max_over(uint32_t x) {
  x = max(x, moved<kSwapOne>(x));
  x = max(x, moved<kSwapTwo>(x));
  if constexpr (LANES >= 8) x = max(x, moved<kMirrorEight>(x));
  if constexpr (LANES == 16) x = max(x, moved<kMirror>(x));
  return x;
}

// x / s rounded to the nearest code for eight values of a run: ties to the even code, saturating (Sec. 2.1).  A quotient that lies on a
// tie is exact after the correction by its remainder, and others are further from one than the error of 2^-22.
__device__ __forceinline__ uint32_t eight_codes(u4 x, float s, bool finite) {
  const float r = __builtin_amdgcn_rcpf(s);
  uint32_t code = 0;
  auto quotient = [&](_Float16 h) {
    const float a = (float)h;
    float u = a * r;
    u = __builtin_fmaf(__builtin_fmaf(-u, s, a), r, u);  // also -0 to 0: the sign of a code is (x < 0)
    return __builtin_amdgcn_fmed3f(u, -6.0f, 6.0f);
  };
  const h2 p0 = halves(x[0]), p1 = halves(x[1]), p2 = halves(x[2]), p3 = halves(x[3]);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, quotient(p0[0]), quotient(p0[1]), 1.0f, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, quotient(p1[0]), quotient(p1[1]), 1.0f, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, quotient(p2[0]), quotient(p2[1]), 1.0f, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, quotient(p3[0]), quotient(p3[1]), 1.0f, 3);
  return finite ? code : 0;
}

// Scale of a run from the bits of its largest magnitude: fp16(max / 6), 1 where that is 0, at most 10912 = fp16's largest value / 6
// rounded down (a finite run stays finite), NaN for a run that holds an inf or a NaN.
__device__ __forceinline__ _Float16 scale_of(uint32_t most) {
  const _Float16 s = (_Float16)((float)__builtin_bit_cast(_Float16, (uint16_t)most) / 6.0f);
  if (most >= 0x7C00u) return __builtin_bit_cast(_Float16, (uint16_t)0x7E00);
  return s == (_Float16)0 ? (_Float16)1 : s > (_Float16)10912 ? (_Float16)10912 : s;
}

struct RowsArgs {
  View v;
  uint16_t *k, *v_rows;
  int64_t k_stride, k_head, v_stride, v_head;
  int vec;  // rows are 16-byte aligned
};

// Tiles of a workgroup: of several heads, whose rows lie beside each other.
constexpr int kWaves = 4;

// A wavefront has 64 / (D / 8) tokens at a time, eight channels of one of them to a lane; all of its rows are asked for before the page
// is looked up.  The tile's planes are put together in LDS, in the cache's order, and leave as whole words; a word of V's codes holds four
// tokens and goes byte by byte where some of them are not this call's.
template <int D, int G>
__global__ __launch_bounds__(64 * kWaves) void write_kernel(RowsArgs a) {
  constexpr int RUNS = D / G, CHUNKS = D / 8, W = Lane<D>::W, CODES = 8 * D, SCALES = kTile * RUNS * 2, PASSES = kTile * CHUNKS / 64, TOKENS = 64 / CHUNKS;
  __shared__ __align__(16) uint8_t image[kWaves][2 * (CODES + SCALES)];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = lane_id();
  const int unit = blockIdx.x * kWaves + wave, item = (int)a.v.heads.quotient(unit), head = unit - item * a.v.kv_heads;
  TileRows t;
  if (!tile_rows(a.v, item, &t) || t.tile < 0) return;
  const int c = lane % CHUNKS;
  u4 x[PASSES][2];
#pragma unroll
  for (int i = 0; i < PASSES; i++) {
    const int token = i * TOKENS + lane / CHUNKS;
    x[i][0] = x[i][1] = u4{0, 0, 0, 0};
    if (token >= t.first && token < t.end) {
      const int64_t row = t.row + token;
      x[i][0] = load8(a.k + row * a.k_stride + head * a.k_head + 8 * c, a.vec);
      x[i][1] = load8(a.v_rows + row * a.v_stride + head * a.v_head + 8 * c, a.vec);
    }
  }
  int in_page;
  uint8_t* const block = block_of(a.v, t.b, t.tile, head, &in_page);
  if (!block) return;
  uint8_t* const img = image[wave];
#pragma unroll
  for (int i = 0; i < PASSES; i++) {
    if ((i + 1) * TOKENS <= t.first || i * TOKENS >= t.end) continue;
    const int token = i * TOKENS + lane / CHUNKS, word = c / 4, run = c * 8 / G;
    uint32_t code[2];
#pragma unroll
    for (int which = 0; which < 2; which++) {
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 4; j++) most = max_halves(most, x[i][which][j] & 0x7FFF7FFFu);
      most = max_over<G / 8>(max(most & 0xFFFFu, most >> 16));
      const _Float16 s = scale_of(most);
      code[which] = eight_codes(x[i][which], (float)s, most < 0x7C00u);
      if (c * 8 % G == 0) *(_Float16*)(img + 2 * CODES + which * SCALES + 2 * (which ? (token / 4 * RUNS + run) * 4 + token % 4 : token * RUNS + run)) = s;
    }
    *(uint32_t*)(img + word / W * 256 * W + ((c & 3) * 16 + token) * 4 * W + word % W * 4) = code[0];
    // V: channels 8 (c & 1) .. + 7 of 32 word + 16 (c >> 1 & 1): joined with the other half's codes, in the lane two further, and each of the
    // two lanes stores four channels, the lower one the first four.
    const uint32_t other = moved<kSwapTwo>(code[1]);
    const bool upper = (c & 2) != 0;
    uint32_t low = upper ? other : code[1], high = upper ? code[1] : other;  // a, b
    if (upper) low >>= 16, high >>= 16;
    const uint32_t first = token & 1 ? high : low, second = token & 1 ? low : high;  // in the lower and the upper nibble
    const uint32_t even = (first & 0x0F0Fu) | (second & 0x0F0Fu) << 4, odd = (first >> 4 & 0x0F0Fu) | (second & 0xF0F0u);
    uint8_t* const to = img + CODES + word / W * 256 * W + (token / 4 * 16 + (c & 1) * 8 + (upper ? 4 : 0)) * 4 * W + word % W * 4 + token % 4;
    to[0] = (uint8_t)even, to[4 * W] = (uint8_t)odd, to[8 * W] = (uint8_t)(even >> 8), to[12 * W] = (uint8_t)(odd >> 8);
  }
  wave_sync();
  uint8_t* const kc = block + in_page * CODES;
  uint8_t* const vc = kc + a.v.codes;
  uint8_t* const ks = block + 2 * a.v.codes + in_page * SCALES;
  uint8_t* const vs = ks + a.v.scales;
  auto there = [&](int token) { return token >= t.first && token < t.end; };
  if (t.first == 0 && t.end == kTile) {
    for (int o = lane * 16; o < CODES; o += 1024) {
      *(u4*)(kc + o) = *(const u4*)(img + o);
      *(u4*)(vc + o) = *(const u4*)(img + CODES + o);
    }
    for (int o = lane * 4; o < SCALES; o += 256) {
      *(uint32_t*)(ks + o) = *(const uint32_t*)(img + 2 * CODES + o);
      *(uint32_t*)(vs + o) = *(const uint32_t*)(img + 2 * CODES + SCALES + o);
    }
    return;
  }
  for (int o = lane * 4; o < CODES; o += 256) {
    if (there(o / (4 * W) % 16)) *(uint32_t*)(kc + o) = *(const uint32_t*)(img + o);
    const int token = o / (64 * W) % 4 * 4;
    if (there(token) && there(token + 3)) {
      *(uint32_t*)(vc + o) = *(const uint32_t*)(img + CODES + o);
    } else {
      for (int j = 0; j < 4; j++)
        if (there(token + j)) vc[o + j] = img[CODES + o + j];
    }
  }
  for (int o = lane * 2; o < SCALES; o += 128) {
    if (there(o / (2 * RUNS))) *(uint16_t*)(ks + o) = *(const uint16_t*)(img + 2 * CODES + o);
    if (there(o / (8 * RUNS) * 4 + o / 2 % 4)) *(uint16_t*)(vs + o) = *(const uint16_t*)(img + 2 * CODES + SCALES + o);
  }
}

template <int D, int G>
__global__ __launch_bounds__(64 * kWaves) void read_kernel(RowsArgs a) {
  constexpr int RUNS = D / G, W = Lane<D>::W, CODES = 8 * D, SCALES = kTile * RUNS * 2, ROW = D + 8;
  __shared__ __align__(16) _Float16 image[kWaves][kTile * ROW];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = lane_id();
  const int unit = blockIdx.x * kWaves + wave, item = (int)a.v.heads.quotient(unit), head = unit - item * a.v.kv_heads;
  TileRows t;
  if (!tile_rows(a.v, item, &t)) return;
  int in_page = 0;
  const uint8_t* const block = t.tile < 0 ? nullptr : block_of(a.v, t.b, t.tile, head, &in_page);
  auto there = [&](int token) { return token >= t.first && token < t.end; };
  auto row_of = [&](uint16_t* p, int64_t stride, int64_t h, int token) { return p + (int64_t)(t.row + token) * stride + head * h; };
  if (!block) {
    for (int u = lane; u < kTile * D / 8; u += 64) {
      const int token = u / (D / 8), c = u % (D / 8);
      if (!there(token)) continue;
      store8(row_of(a.k, a.k_stride, a.k_head, token) + 8 * c, u4{0, 0, 0, 0}, a.vec);
      store8(row_of(a.v_rows, a.v_stride, a.v_head, token) + 8 * c, u4{0, 0, 0, 0}, a.vec);
    }
    return;
  }
  const int g = lane >> 4, c = lane & 15;
  const uint8_t* const kc = block + in_page * CODES;
  const uint8_t* const ks = block + 2 * a.v.codes + in_page * SCALES;
  Lane<D> kw, vw;
  kw.load(kc, lane);
  vw.load(kc + a.v.codes, lane);
  Scales<RUNS> sk;
  sk.load(ks + c * RUNS * 2);
  Scales<4 * RUNS> sv;
  sv.load(ks + a.v.scales + g * RUNS * 8);
  _Float16* const img = image[wave];
#pragma unroll
  for (int i = 0; i < Lane<D>::kWords; i++) *(u4*)(img + c * ROW + 32 * i + 8 * g) = __builtin_bit_cast(u4, restore_k(kw.w[i], sk.twice(32 * i / G)));
  wave_sync();
#pragma unroll
  for (int u = lane; u < kTile * D / 8; u += 64) {
    const int token = u / (D / 8), part = u % (D / 8);
    if (there(token)) store8(row_of(a.k, a.k_stride, a.k_head, token) + 8 * part, *(const u4*)(img + token * ROW + 8 * part), a.vec);
  }
  wave_sync();
#pragma unroll
  for (int i = 0; i < Lane<D>::kWords; i++) {
    const int run = 32 * i / G * 2;
    u2 x, y;
    restore_v(vw.w[i], sv.w[run], sv.w[run + 1], &x, &y);
    const h4 xs = __builtin_bit_cast(h4, x), ys = __builtin_bit_cast(h4, y);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      img[(4 * g + j) * ROW + 32 * i + c] = xs[j];
      img[(4 * g + j) * ROW + 32 * i + 16 + c] = ys[j];
    }
  }
  wave_sync();
  for (int u = lane; u < kTile * D / 8; u += 64) {
    const int token = u / (D / 8), part = u % (D / 8);
    if (there(token)) store8(row_of(a.v_rows, a.v_stride, a.v_head, token) + 8 * part, *(const u4*)(img + token * ROW + 8 * part), a.vec);
  }
}

template <bool WRITE>
int run_rows(const ams_kv_cache* cache, int64_t rows, uint16_t* k, uint16_t* v, int64_t k_stride, int64_t k_head, int64_t v_stride, int64_t v_head, void* stream) {
  RowsArgs a;
  if (const int rc = make_view(cache, rows, &a.v); rc != AMS_OK) return rc;
  if (rows > 0 && (!k || !v)) return AMS_ERR_NULL;
  if (!aligned(k, 2) || !aligned(v, 2)) return AMS_ERR_ALIGN;
  const int64_t units = (cache->q_starts ? rows / kTile + 2 * (int64_t)cache->batch : cache->batch) * cache->kv_heads, grid = (units + kWaves - 1) / kWaves;
  if (rows > 0 && !launchable(grid, 64 * kWaves)) return AMS_ERR_SHAPE;
  if (const int rc = device_status(); rc != AMS_OK) return rc;
  if (rows == 0 || cache->batch == 0) return AMS_OK;
  a.k = k, a.v_rows = v, a.k_stride = k_stride, a.k_head = k_head, a.v_stride = v_stride, a.v_head = v_head;
  a.vec = aligned(k, 16) && aligned(v, 16) && (k_stride | k_head | v_stride | v_head) % 8 == 0;
  auto go = [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    if constexpr (WRITE)
      hipLaunchKernelGGL((write_kernel<D, G>), dim3((unsigned)grid), dim3(64 * kWaves), 0, (hipStream_t)stream, a);
    else
      hipLaunchKernelGGL((read_kernel<D, G>), dim3((unsigned)grid), dim3(64 * kWaves), 0, (hipStream_t)stream, a);
  };
  dispatch(cache->head_dim, cache->scale_group, go);
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

bool load_cache() { return loaded((const void*)write_kernel<64, 32>); }

bool aligned(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

static bool sizes_ok(int kv_heads, int head_dim, int page_size, int scale_group) {
  if (kv_heads < 1 || kv_heads > AMS_KV_MAX_HEADS || page_size < kTile || page_size % kTile || page_size > AMS_KV_MAX_PAGE) return false;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return false;
  return (scale_group == 32 || scale_group == 64 || scale_group == 128) && scale_group <= head_dim;
}

int make_view(const ams_kv_cache* c, int64_t rows, View* v) {
  if (!c || !c->pages || (c->batch > 0 && (!c->block_table || !c->kv_lens))) return AMS_ERR_NULL;
  if (!sizes_ok(c->kv_heads, c->head_dim, c->page_size, c->scale_group)) return AMS_ERR_SHAPE;
  if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFF || c->batch < 0 || c->batch > AMS_KV_MAX_BATCH || c->table_width < 1 || c->table_stride < 0) return AMS_ERR_SHAPE;
  if ((int64_t)c->table_width * c->page_size > AMS_KV_MAX_TOKENS || rows < 0 || rows > AMS_KV_MAX_TOKENS) return AMS_ERR_SHAPE;
  if (!c->q_starts && rows != c->batch) return AMS_ERR_SHAPE;
  if (!aligned(c->pages, 16) || !aligned(c->block_table, 4) || !aligned(c->kv_lens, 4) || !aligned(c->q_starts, 4)) return AMS_ERR_ALIGN;
  const Planes p = planes(c->head_dim, c->page_size, c->scale_group);
  v->pages = (uint8_t*)c->pages, v->table = c->block_table, v->lens = c->kv_lens, v->starts = c->q_starts;
  v->table_stride = c->table_stride, v->page_bytes = (int64_t)c->kv_heads * p.block;
  v->n_pages = (int)c->n_pages, v->table_width = c->table_width, v->batch = c->batch, v->kv_heads = c->kv_heads, v->rows = (int)rows;
  v->page_tiles = divisor((uint32_t)(c->page_size / kTile)), v->heads = divisor((uint32_t)c->kv_heads), v->page_size = c->page_size, v->codes = p.codes, v->scales = p.scales, v->block = p.block;
  return AMS_OK;
}

}  // namespace ams_kv

extern "C" {

int ams_kv_block_bytes(int head_dim, int page_size, int scale_group, size_t* bytes) {
  if (!bytes) return AMS_ERR_NULL;
  if (!ams_kv::sizes_ok(1, head_dim, page_size, scale_group)) return AMS_ERR_SHAPE;
  *bytes = (size_t)ams_kv::planes(head_dim, page_size, scale_group).block;
  return AMS_OK;
}

int ams_kv_write(const ams_kv_cache* cache, const uint16_t* K, const uint16_t* V, int64_t rows, int64_t k_stride, int64_t k_head_stride, int64_t v_stride,
                 int64_t v_head_stride, void* stream) {
  return ams_kv::run_rows<true>(cache, rows, (uint16_t*)K, (uint16_t*)V, k_stride, k_head_stride, v_stride, v_head_stride, stream);
}

int ams_kv_read(const ams_kv_cache* cache, uint16_t* K, uint16_t* V, int64_t rows, int64_t k_stride, int64_t k_head_stride, int64_t v_stride,
                int64_t v_head_stride, void* stream) {
  return ams_kv::run_rows<false>(cache, rows, K, V, k_stride, k_head_stride, v_stride, v_head_stride, stream);
}

}  // extern "C"
