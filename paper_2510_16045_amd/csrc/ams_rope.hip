// Rotary positions: rows of Q and K rotated by their positions, pair by pair.
//
//   y_a = m (x_a cos t - x_b sin t),  y_b = m (x_b cos t + x_a sin t),  t = p w_i
//
// for pair i of a head's first `rotary_dim` channels: a, b = i, i + rotary_dim / 2, or 2 i, 2 i + 1 where they are interleaved.
//
// The angle.  w_i is given as a fraction of a turn in 64-bit fixed point, off by what the host's 53 bits leave (some 2^-54 turns for the fastest
// pairs); p times that modulo 2^64 is the angle modulo a turn, off by p 2^-54 turns, at p = 131072 by 5e-11 radians, where a product of
// 32-bit floats is off by 0.008.  Its upper 32 bits (to 1.5e-9 radians; the product's lowest word is left out) are reduced to an eighth of a turn on either side of a quarter, where sin and cos are polynomials: the Taylor series up to x^9 and
// x^8, whose next terms are below 2e-9 and 3e-8.  So there is no table of cosines to read, and no longest position.
//
// What bounds it: memory, and a launch where there are few rows.  16384 rows of 72 heads of 128: 604 MB in 118 us, 5.1 TB/s, a copy's rate; in
// place 126; 3104 rows of 32 heads of 256 of which 64 channels are rotated 26.7 (4.6 TB/s), in place, where only those move, 8.8.  A wavefront
// works its angles out once (some 40 operations a pair) for all heads that it takes, eight heads at a time of 128 channels; 8192
// wavefronts (4096: the ragged rows 34 us instead of 25.5, 16384 27).
#include "ams_kv.h"

#include <float.h>
#include <math.h>

#include <algorithm>

namespace ams_kv {

struct RopeTensor {
  const uint16_t* in;
  uint16_t* out;
  int64_t in_stride, in_head, out_stride, out_head;
};
struct RopeArgs {
  RopeTensor q, k;
  const uint64_t* turns;
  const int32_t *positions, *lens, *starts;
  int64_t rows, first_row;  // first_row: of the launch
  float magnitude;
  int batch, heads, all_heads;  // heads: of q; all_heads: with k's behind them
  int pairs, rest;              // of a head: pairs, and channels behind them that are copied (0 where they are in place)
  int chunks;                   // of a head: what one lane takes of it at a time
  int at_once;                  // heads that a wavefront takes at a time
  int passes;                   // of a wavefront
  Divisor by_chunks, by_parts;  // parts: wavefronts of a row
  int interleaved, transposed;
};

// The position of a row, the wavefront's own: false where no sequence has it.  Row starts count as in [0, rows], as the cache's calls take them.
__device__ __forceinline__ bool row_position(const RopeArgs& a, int64_t row, int* position) {
  if (a.positions) {
    *position = a.positions[row];
    return true;
  }
  if (!a.starts) {
    if (row >= a.batch) return false;
    *position = max(a.lens[row], 0) - 1;
    return true;
  }
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = min(b0 + lane_id(), a.batch - 1);
    const int first = a.starts[b], end = min(max(a.starts[b + 1], 0), (int)a.rows), len = max(a.lens[b], 0);
    const unsigned long long found = __ballot(first <= row && row < end);
    if (found) {
      *position = (int)((uint32_t)__builtin_amdgcn_readlane(len, __builtin_ctzll(found)) - (uint32_t)__builtin_amdgcn_readlane(end, __builtin_ctzll(found)) + (uint32_t)row);
      return true;
    }
  }
  return false;
}

// cos and sin of p times `turn`.
__device__ __forceinline__ void angle(uint64_t turn, int p, float magnitude, int transposed, float* c, float* s) {
  const uint32_t low = (uint32_t)turn, high = (uint32_t)(turn >> 32);
  uint32_t at = (uint32_t)p * high + __umulhi((uint32_t)p, low);  // of a turn, in 2^-32
  if (p < 0) at -= low;
  const uint32_t quarter = (at + (1u << 29)) >> 30;
  const float x = (float)(int)(at - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi 2^-32
  const float xx = x * x;
  const float sine = x + x * xx * (-1.0f / 6 + xx * (1.0f / 120 + xx * (-1.0f / 5040 + xx * (1.0f / 362880))));
  const float cosine = 1.0f + xx * (-0.5f + xx * (1.0f / 24 + xx * (-1.0f / 720 + xx * (1.0f / 40320))));
  const float y = quarter & 1 ? cosine : sine;
  float z = quarter & 1 ? sine : cosine;
  if ((quarter + 1) & 2) z = -z;
  *c = magnitude * z;
  *s = magnitude * (((quarter >> 1) ^ (uint32_t)transposed) & 1 ? -y : y);
}

__device__ __forceinline__ void turn_pair(_Float16& a, _Float16& b, float c, float s) {
  const float x = (float)a, y = (float)b;
  a = (_Float16)(x * c - y * s);
  b = (_Float16)(y * c + x * s);
}

// VEC values that lie together.
template <int VEC>
struct Piece {
  typedef _Float16 Values __attribute__((ext_vector_type(VEC)));
  Values x;
  // STREAMED: what is read once and written once stays out of the caches.
  template <bool STREAMED>
  __device__ __forceinline__ void load(const uint16_t* from) {
    x = STREAMED ? __builtin_nontemporal_load((const Values*)from) : *(const Values*)from;
  }
  template <bool STREAMED>
  __device__ __forceinline__ void store(uint16_t* to) const {
    if constexpr (STREAMED)
      __builtin_nontemporal_store(x, (Values*)to);
    else
      *(Values*)to = x;
  }
};

// A wavefront takes heads of one row, `at_once` of them side by side; its lanes keep their angles for all of them.  A lane has pieces of
// VEC channels: two where they are halves of pairs, one of neighbours or of channels that are copied.
template <int VEC, bool INTERLEAVED, bool STREAMED>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int PAIRS = INTERLEAVED && VEC > 1 ? VEC / 2 : VEC;
  const int lane = lane_id();
  const uint32_t unit = blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const uint32_t of_launch = a.by_parts.quotient(unit), part = unit - of_launch * a.by_parts.by;
  const int64_t row = a.first_row + of_launch;
  if (row >= a.rows) return;
  int position;
  if (!row_position(a, row, &position)) return;
  const int turned = a.pairs / PAIRS;  // of the chunks
  const int sub = (int)a.by_chunks.quotient((uint32_t)lane), first_head = (int)part * a.passes * a.at_once + sub;
  if (sub >= a.at_once) return;
  for (int chunk = lane - sub * a.chunks; chunk < a.chunks; chunk += 64) {
    float c[PAIRS], s[PAIRS];
    if (chunk < turned) {
#pragma unroll
      for (int i = 0; i < PAIRS; i++) angle(a.turns[chunk * PAIRS + i], position, a.magnitude, a.transposed, &c[i], &s[i]);
    }
    for (int pass = 0; pass < a.passes; pass++) {
      const int head = first_head + pass * a.at_once;
      if (head >= a.all_heads) break;
      const RopeTensor& t = head < a.heads ? a.q : a.k;
      const int h = head < a.heads ? head : head - a.heads;
      const uint16_t* const in = t.in + row * t.in_stride + (int64_t)h * t.in_head;
      uint16_t* const out = t.out + row * t.out_stride + (int64_t)h * t.out_head;
      Piece<VEC> x, y;
      if (chunk >= turned) {
        const int at = 2 * a.pairs + (chunk - turned) * VEC;
        x.template load<STREAMED>(in + at);
        x.template store<STREAMED>(out + at);
      } else if constexpr (INTERLEAVED && VEC > 1) {
        x.template load<STREAMED>(in + chunk * VEC);
#pragma unroll
        for (int i = 0; i < PAIRS; i++) {
          _Float16 p = x.x[2 * i], q = x.x[2 * i + 1];
          turn_pair(p, q, c[i], s[i]);
          x.x[2 * i] = p, x.x[2 * i + 1] = q;
        }
        x.template store<STREAMED>(out + chunk * VEC);
      } else {
        const int i = INTERLEAVED ? 2 * chunk : VEC * chunk, j = INTERLEAVED ? i + 1 : i + a.pairs;
        x.template load<STREAMED>(in + i), y.template load<STREAMED>(in + j);
#pragma unroll
        for (int k = 0; k < VEC; k++) {
          _Float16 p = x.x[k], q = y.x[k];
          turn_pair(p, q, c[k], s[k]);
          x.x[k] = p, y.x[k] = q;
        }
        x.template store<STREAMED>(out + i), y.template store<STREAMED>(out + j);
      }
    }
  }
}

bool load_rope() { return loaded((const void*)rope_kernel<8, false, false>); }

}  // namespace ams_kv

using namespace ams_kv;

extern "C" {

int ams_rope_frequencies(int rotary_dim, double base, int scaling, double factor, int64_t trained_len, uint64_t* turns, float* magnitude) {
  if (!turns || !magnitude) return AMS_ERR_NULL;
  if (rotary_dim < 2 || rotary_dim > AMS_ROPE_MAX_DIM || rotary_dim % 2 || !(base >= 1) || !(base <= 1e30)) return AMS_ERR_SHAPE;
  if (scaling < AMS_ROPE_PLAIN || scaling > AMS_ROPE_YARN) return AMS_ERR_SHAPE;
  if (scaling != AMS_ROPE_PLAIN && (!(factor >= 1) || !(factor <= 1e9))) return AMS_ERR_SHAPE;
  if ((scaling == AMS_ROPE_BANDS || scaling == AMS_ROPE_YARN) && (trained_len < 1 || trained_len > INT32_MAX)) return AMS_ERR_SHAPE;
  if (scaling == AMS_ROPE_YARN && !(base > 1)) return AMS_ERR_SHAPE;
  constexpr double kTurn = 6.283185307179586476925;
  const double r = rotary_dim, len = (double)trained_len;
  if (scaling == AMS_ROPE_NTK && rotary_dim > 2) base *= pow(factor, r / (r - 2));
  double lo = 0, hi = 0;
  if (scaling == AMS_ROPE_YARN) {  // the pair that makes n turns within the trained length
    auto pair = [&](double n) { return r * log(len / (kTurn * n)) / (2 * log(base)); };
    lo = std::max(floor(pair(32)), 0.0), hi = std::min(ceil(pair(1)), r - 1);
  }
  for (int i = 0; i < rotary_dim / 2; i++) {
    double w = pow(base, -2.0 * i / r), kept = 1;
    if (scaling == AMS_ROPE_LINEAR) kept = 0;
    if (scaling == AMS_ROPE_BANDS) kept = std::min(1.0, std::max(0.0, (len * w / kTurn - 1) / 3));
    if (scaling == AMS_ROPE_YARN) kept = 1 - std::min(1.0, std::max(0.0, (i - lo) / std::max(hi - lo, 0.001)));
    if (kept < 1) w = kept * w + (1 - kept) * w / factor;
    turns[i] = (uint64_t)ldexp(w / kTurn, 64);  // below a sixth of a turn
  }
  *magnitude = scaling == AMS_ROPE_YARN ? (float)(0.1 * log(factor) + 1) : 1.0f;
  return AMS_OK;
}

int ams_rope(const ams_rotation* rotation, const ams_rope_rows* Q, const ams_rope_rows* K, int64_t rows, int head_dim, void* stream) {
  if (!rotation || !Q) return AMS_ERR_NULL;
  const ams_rotation& r = *rotation;
  if (rows < 0 || rows > AMS_KV_MAX_TOKENS || head_dim < 1 || head_dim > AMS_ROPE_MAX_DIM || r.rotary_dim < 2 || r.rotary_dim % 2 || r.rotary_dim > head_dim) return AMS_ERR_SHAPE;
  if (Q->heads < 1 || Q->heads > AMS_KV_MAX_HEADS || (K && (K->heads < 1 || K->heads > AMS_KV_MAX_HEADS)) || r.batch < 0 || r.batch > AMS_KV_MAX_BATCH) return AMS_ERR_SHAPE;
  if (!(fabsf(r.magnitude) <= FLT_MAX) || (!r.positions && !r.q_starts && rows != r.batch)) return AMS_ERR_SHAPE;
  if (!r.turns || (rows > 0 && (!Q->in || !Q->out || (K && (!K->in || !K->out)))) || (!r.positions && r.batch > 0 && !r.kv_lens)) return AMS_ERR_NULL;
  if (!aligned(r.turns, 8) || !aligned(r.positions, 4) || !aligned(r.kv_lens, 4) || !aligned(r.q_starts, 4)) return AMS_ERR_ALIGN;
  bool in_place = true;
  // what a lane may take at once, in values: as many as divide the pairs (neighbours: the rotated channels), the strides and, in bytes, the addresses
  uint64_t common = r.interleaved ? r.rotary_dim : r.rotary_dim / 2;
  for (const ams_rope_rows* t : {Q, K}) {
    if (!t) continue;
    if (!aligned(t->in, 2) || !aligned(t->out, 2)) return AMS_ERR_ALIGN;
    common |= (uintptr_t)t->in / 2 | (uintptr_t)t->out / 2 | (uint64_t)(t->in_stride | t->in_head_stride | t->out_stride | t->out_head_stride);
    in_place = in_place && t->in == t->out && t->in_stride == t->out_stride && t->in_head_stride == t->out_head_stride;
  }
  if (const int rc = device_status(); rc != AMS_OK) return rc;
  if (rows == 0 || (!r.positions && r.batch == 0)) return AMS_OK;
  RopeArgs a = {};
  a.q = {Q->in, Q->out, Q->in_stride, Q->in_head_stride, Q->out_stride, Q->out_head_stride};
  if (K) a.k = {K->in, K->out, K->in_stride, K->in_head_stride, K->out_stride, K->out_head_stride};
  a.turns = r.turns, a.positions = r.positions, a.lens = r.kv_lens, a.starts = r.q_starts, a.rows = rows, a.magnitude = r.magnitude;
  a.batch = r.batch, a.heads = Q->heads, a.all_heads = Q->heads + (K ? K->heads : 0);
  a.pairs = r.rotary_dim / 2, a.rest = in_place ? 0 : head_dim - r.rotary_dim;
  common |= (uint64_t)a.rest;
  const int vec = common % 8 == 0 ? 8 : common % 4 == 0 ? 4 : common % 2 == 0 ? 2 : 1;
  a.chunks = a.pairs / (r.interleaved && vec > 1 ? vec / 2 : vec) + a.rest / vec;
  // Where a wavefront's stores fill whole lines of 128 bytes and the rows are more than the caches hold for whoever reads them next: past the
  // caches (16384 rows of 72 heads of 128 125 -> 116 us, 3104 of 32 of 256 25.5 -> 23.0; 2048 of 40 of 128 11.3 and 11.5; lines in parts,
  // 8000 rows of 40 heads of 80, 28 -> 36).
  const bool streamed = vec == 8 && (r.interleaved ? r.rotary_dim : r.rotary_dim / 2) % 64 == 0 && a.rest % 64 == 0 && rows * (Q->heads + (K ? K->heads : 0)) * head_dim >= (int64_t)16 << 20;
  a.at_once = std::max(64 / a.chunks, 1);
  const int64_t turns = (a.all_heads + a.at_once - 1) / a.at_once;
  constexpr int64_t kWavefronts = 8192;
  const int64_t parts = std::min(std::max<int64_t>(kWavefronts / rows, 1), turns);
  a.passes = (int)((turns + parts - 1) / parts);
  a.by_chunks = divisor((uint32_t)a.chunks), a.by_parts = divisor((uint32_t)((turns + a.passes - 1) / a.passes));
  a.interleaved = r.interleaved != 0, a.transposed = r.transposed != 0;
  // One launch has fewer than 2^32 threads (of more the runtime leaves out what passes that, with no error).
  constexpr int64_t kLaunchRows = 1 << 25;  // of a wavefront each
  static_assert(kLaunchRows >= kWavefronts, "more rows have no parts");
  auto launch = [&](auto kernel) {
    for (a.first_row = 0; a.first_row < rows; a.first_row += kLaunchRows)
      hipLaunchKernelGGL(kernel, dim3((unsigned)((std::min(rows - a.first_row, kLaunchRows) * a.by_parts.by + 3) / 4)), dim3(256), 0, (hipStream_t)stream, a);
  };
  auto of_layout = [&](auto interleaved) {
    constexpr bool I = decltype(interleaved)::value;
    if (streamed) return launch(rope_kernel<8, I, true>);
    if (vec == 8) return launch(rope_kernel<8, I, false>);
    if (vec == 4) return launch(rope_kernel<4, I, false>);
    if (vec == 2) return launch(rope_kernel<2, I, false>);
    launch(rope_kernel<1, I, false>);
  };
  r.interleaved ? of_layout(Int<1>()) : of_layout(Int<0>());
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

}  // extern "C"
