// Attention over the 4-bit KV cache: the entry points, and which kernel and how many workgroups a call gets.
#include "ams_kv_attention.h"

#include <float.h>
#include <stdio.h>

#include <algorithm>

namespace ams_kv {

// ---- launch ------------------------------------------------------------------------------------------
constexpr int kComputeUnits = 256;
// The host knows no lengths: keys are what the block table has room for, and the figures here are those of tables as wide as the longest
// sequence.  In tables for 131072 tokens 64 sequences of up to 1000 get four wavefronts (13.0 us, in their own 11.7), four prompts of 1024
// tiles of 256 rows (72, 66), 1536 rows of 16 heads stream_kernel (52, 44).
// Rows of a kv head that stream_kernel takes in one tile.  Beyond them it reads the cache once for every 64, where tile_kernel restores
// it once for 128 or 256 rows.
constexpr int kStreamRows = 64;
// Tiles of 128 rows: with fewer stream_kernel, which shares keys out evenly, is faster than tiles that do not fill the chip, or of different
// lengths: 32 query and 8 kv heads of 128, one sequence of 8192: 128 tiles 100 us, tile_kernel 193; 256 tiles 170 and 198; 384 252 and
// 257; lengths of 819 to 8192, 432 tiles 219 and 264; 8 of 4096, 400 tiles 235 and 241, 512 193 and 156; 256 channels, 8 of up to 4096, 280
// tiles 165 and 222, 440 235 and 270, but one of 8192, 256 tiles, 335 and 313.  With fewer keys the shares fit less well (16 heads, 2048
// keys: 128 tiles 34 and 56, 160 58 and 55, 192 64 and 57, 256 54 and 59).  Keys of kUncutSteps steps are never shared out.
constexpr int kFewTiles = 448, kFewShortTiles = 160;  // with kLongKeys keys or more, and with fewer
// Tiles of 16 rows of stream_kernel: so many or fewer have eight wavefronts (one sequence of 131071, 8 kv heads: 42 -> 38 us).
constexpr int kLoneTiles = 64;
// So have up to 256 tiles with so many keys at most (64 x 1000, 4 kv heads: 14.4 -> 12.1 us; 32 ragged x 8192, 8 heads: 42 -> 46).
constexpr int kShortKeys = 4096;
// Keys from which on tiles of 256 rows, which restore a key once for twice the rows, are the faster ones where they fill the chip (2048 rows
// over 8192 keys: 267 us, tiles of 128 285); with fewer the shorter tiles end more evenly (4 times 1024 over 1024: 76 and 69; a window of
// 512: 64 and 54).
constexpr int kLongKeys = 4096;
constexpr size_t kCountBytes = 64 * 1024;  // of a workspace: counts of any call (2 kv_heads x shares of them), at its front
static_assert(8 * kComputeUnits * sizeof(uint32_t) <= kCountBytes && 2 * AMS_KV_MAX_HEADS * sizeof(uint32_t) <= kCountBytes, "two for each share of each head");

struct Plan {
  bool tile;  // tile_kernel
  int waves;  // of its workgroups
  int qt, rows, part_rows;
  int64_t row_tiles;  // at most so many over all sequences
  int64_t shares;
  bool cut;
  size_t workspace;   // bytes that this many shares need
};
Plan make_plan(const ams_kv_cache* c, int64_t rows, int heads, int64_t max_q_len, int64_t window, size_t workspace) {
  Plan p;
  const int R = heads / c->kv_heads;
  const int64_t most = (c->q_starts ? std::min(max_q_len > 0 ? max_q_len : rows, rows) : 1) * R;
  const int64_t capacity = (int64_t)c->table_width * c->page_size, keys = window > 0 ? std::min(window, capacity) : capacity;
  // column tiles of 16 rows: as few as hold them (40 rows of 16 sequences of 3001, 8 kv heads: three 33 us, four 38)
  p.qt = most <= 16 ? 1 : most <= 32 || c->head_dim == 256 ? 2 : most <= 48 ? 3 : 4;
  const int64_t tiles = rows * R / 128 * c->kv_heads;
  p.tile = most > kStreamRows && (tiles >= (keys < kLongKeys ? kFewShortTiles : kFewTiles) || keys <= kUncutSteps * kStep);
  p.waves = 4;
  if (p.tile && c->head_dim < 256 && tiles >= 2 * kComputeUnits && keys >= kLongKeys) p.waves = 8;
  p.rows = p.tile ? 32 * p.waves : 16 * p.qt;
  p.row_tiles = c->q_starts ? rows * R / p.rows + c->batch : c->batch * (int64_t)((R + p.rows - 1) / p.rows);
  // Tiles of stream_kernel, if no sequence has more rows than the caller says: eight wavefronts where they are few, or short and no compute
  // unit has two; with several column tiles of 128 channels wherever no compute unit has two (16 rows of 32 sequences of 1500, 32 query and
  // 8 kv heads: 48 -> 30 us; 64 of one of 131071: 85 -> 70; with two, 64 sequences of 500 and 8 rows: 17 -> 25; 64 channels: 64 rows of one of
  // 131071 51 -> 49, 32 rows 41 -> 46).
  const int64_t about = std::min<int64_t>(p.row_tiles, c->batch * ((most + p.rows - 1) / p.rows)) * c->kv_heads;
  if (!p.tile && p.qt == 1 && c->head_dim < 256 && (about <= kLoneTiles || (about <= kComputeUnits && capacity <= kShortKeys))) p.waves = 8;
  if (!p.tile && p.qt > 1 && c->head_dim == 128 && about <= kComputeUnits) p.waves = 8;
  const int64_t tile_steps = std::max<int64_t>((capacity + kStep - 1) / kStep, 1);
  p.part_rows = (int)std::min<int64_t>(c->q_starts ? std::max<int64_t>(rows, 1) * R : R, p.rows);
  const size_t part = (size_t)c->kv_heads * p.part_rows * (c->head_dim + 4) * sizeof(float);
  const size_t room = std::min<size_t>(workspace, AMS_KV_WORKSPACE_BYTES);
  const int64_t fit = std::max<int64_t>(stream_groups(c->head_dim, p.qt, p.waves) * kComputeUnits / c->kv_heads, 1);
  p.shares = std::min(std::min(fit, p.row_tiles * kMaxParts), room < kCountBytes ? 0 : (int64_t)((room - kCountBytes) / part / 2));
  // A workspace with room for few shares does not pay: whole tiles then, as without one.  From 7/8 of a share to a row tile on, as far as those
  // fit on the chip, equal shares gain more where lengths differ than they lose where they do not: 32 sequences, 32 query and 8 kv heads, of
  // 819 to 8192 tokens whole tiles 85 us, 3 shares 492, 24 74, 29 64, 32 59; all of 8192 whole tiles 90, 3 863, 24 123, 29 105, 32 90.
  p.cut = rows > 0 && !p.tile && p.shares > 1 && 8 * p.shares >= 7 * std::min(fit, p.row_tiles) && tile_steps > kUncutSteps && p.row_tiles * (tile_steps + kTileSteps) <= 0x7FFFFFFF;
  p.workspace = p.cut ? kCountBytes + 2 * (size_t)p.shares * part : 0;
  if (!p.cut) p.shares = p.row_tiles;
  return p;
}

template <typename Args>
static void launch(const Args& a, const Plan& p, const ams_kv_cache* cache, unsigned grid, hipStream_t stream) {
  if (p.tile)
    launch_tile(a, cache->head_dim, cache->scale_group, p.waves, grid, stream);
  else
    launch_stream(a, cache->head_dim, cache->scale_group, p.qt, p.waves, grid, stream);
}

}  // namespace ams_kv

using namespace ams_kv;

extern "C" {

int ams_kv_attention_workspace_bytes(const ams_kv_cache* cache, int64_t rows, int heads, int64_t max_q_len, size_t* bytes) {
  View v;
  if (!bytes) return AMS_ERR_NULL;
  if (const int rc = make_view(cache, rows, &v); rc != AMS_OK) return rc;
  if (heads < 1 || heads % cache->kv_heads || heads > AMS_KV_MAX_HEADS) return AMS_ERR_SHAPE;
  *bytes = make_plan(cache, rows, heads, max_q_len, 0, SIZE_MAX).workspace;
  return AMS_OK;
}

int ams_kv_attention_plan(const ams_kv_cache* cache, int64_t rows, int heads, int64_t window, int64_t max_q_len, size_t workspace_bytes, char* text, size_t text_len) {
  View v;
  if (!text || text_len == 0) return AMS_ERR_NULL;
  if (const int rc = make_view(cache, rows, &v); rc != AMS_OK) return rc;
  if (heads < 1 || heads % cache->kv_heads || heads > AMS_KV_MAX_HEADS || window < 0 || max_q_len < 0 || rows * (heads / cache->kv_heads) > AMS_KV_MAX_TOKENS) return AMS_ERR_SHAPE;
  const Plan p = make_plan(cache, rows, heads, max_q_len, window, workspace_bytes);
  snprintf(text, text_len, "%s rows=%d waves=%d workgroups=%lld shared=%d", p.tile ? "tile" : "stream", p.rows, p.waves, (long long)p.shares * cache->kv_heads, (int)p.cut);
  return AMS_OK;
}

int ams_kv_attention(const ams_kv_cache* cache, const uint16_t* Q, uint16_t* O, float* lse, int64_t rows, int heads, int64_t q_stride, int64_t q_head_stride,
                     int64_t o_stride, int64_t o_head_stride, int64_t lse_stride, float softmax_scale, int causal, int64_t window, int64_t max_q_len,
                     void* workspace, size_t workspace_bytes, void* stream) {
  return ams_kv_attention_scored(cache, nullptr, Q, O, lse, rows, heads, q_stride, q_head_stride, o_stride, o_head_stride, lse_stride, softmax_scale, causal, window, max_q_len, workspace,
                                 workspace_bytes, stream);
}

int ams_kv_attention_scored(const ams_kv_cache* cache, const ams_kv_scores* scores, const uint16_t* Q, uint16_t* O, float* lse, int64_t rows, int heads, int64_t q_stride,
                            int64_t q_head_stride, int64_t o_stride, int64_t o_head_stride, int64_t lse_stride, float softmax_scale, int causal, int64_t window, int64_t max_q_len,
                            void* workspace, size_t workspace_bytes, void* stream) {
  LargeCapArgs a;
  if (const int rc = make_view(cache, rows, &a.v); rc != AMS_OK) return rc;
  if (rows > 0 && (!Q || !O)) return AMS_ERR_NULL;
  if (heads < 1 || heads % cache->kv_heads || heads > AMS_KV_MAX_HEADS || window < 0 || (window > 0 && !causal) || max_q_len < 0 || !(softmax_scale > 0) || !(softmax_scale <= FLT_MAX)) return AMS_ERR_SHAPE;
  if (rows * (heads / cache->kv_heads) > AMS_KV_MAX_TOKENS) return AMS_ERR_SHAPE;
  constexpr float kLog2e = 1.44269504089f;
  const ams_kv_scores none = {nullptr, nullptr, 0}, &x = scores ? *scores : none;
  a.slopes = x.slopes, a.prefixes = x.prefix_lens, a.cap2 = x.softcap * kLog2e, a.to_cap = x.softcap > 0 ? 2 * kLog2e * softmax_scale / x.softcap : 0;
  if (!(x.softcap >= 0) || !(a.cap2 <= FLT_MAX / 4) || !(a.to_cap <= FLT_MAX) || (x.prefix_lens && !causal)) return AMS_ERR_SHAPE;
  if (!aligned(Q, 2) || !aligned(O, 2) || !aligned(lse, 4) || !aligned(workspace, 16) || !aligned(x.slopes, 4) || !aligned(x.prefix_lens, 4)) return AMS_ERR_ALIGN;
  const bool nothing = rows == 0 || cache->batch == 0;
  const Plan p = nothing ? Plan{} : make_plan(cache, rows, heads, max_q_len, window, workspace ? workspace_bytes : 0);
  const int64_t grid = p.shares * cache->kv_heads;
  if (!launchable(grid, 64 * p.waves)) return AMS_ERR_SHAPE;
  if (const int rc = device_status(); rc != AMS_OK) return rc;
  if (nothing) return AMS_OK;
  a.q = Q, a.out = O, a.lse = lse, a.counts = (uint32_t*)workspace, a.parts = (float*)((uint8_t*)workspace + kCountBytes);
  a.q_stride = q_stride, a.q_head = q_head_stride, a.out_stride = o_stride, a.out_head = o_head_stride, a.lse_stride = lse_stride;
  a.scale2 = softmax_scale * kLog2e;
  a.group = heads / cache->kv_heads, a.by_group = divisor((uint32_t)a.group);
  a.causal = causal != 0, a.window = (int)std::min<int64_t>(window, 0x3FFFFFFF);
  a.vec = aligned(Q, 16) && aligned(O, 8) && (q_stride | q_head_stride) % 8 == 0 && (o_stride | o_head_stride) % 4 == 0;
  a.shares = (int)p.shares, a.cut = p.cut, a.row_tiles = (int)p.row_tiles, a.part_rows = p.part_rows;
  if (x.softcap > kLargeCap) {
    a.cap2 = 0, a.cap_of = x.softcap / softmax_scale;
    launch(a, p, cache, (unsigned)grid, (hipStream_t)stream);
  } else if (x.prefix_lens)
    launch<PrefixArgs>(a, p, cache, (unsigned)grid, (hipStream_t)stream);
  else if (x.softcap > 0 || x.slopes)
    launch<ScoredArgs>(a, p, cache, (unsigned)grid, (hipStream_t)stream);
  else
    launch<AttentionArgs>(a, p, cache, (unsigned)grid, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

}  // extern "C"
