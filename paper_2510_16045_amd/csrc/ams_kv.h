// The paged 4-bit KV cache: its layout, what a call says of it, and the device code that its kernels share.
//
// A run of `scale_group` channels of one token and head is held as FP4-e2m1 codes (Sec. 2.2) with one fp16 scale (Eq. 1, "any
// granularity", Sec. 5).  The pool is uint8 [n_pages][kv_heads][block]; a block holds page_size tokens of a head in tiles of 16,
// and lies in four planes: K codes, V codes, K scales, V scales.  A tile's codes are arranged as the lanes of a 64-wide wavefront
// feed them to 16x16x32 fp16 MFMA tiles, W = min(4, D / 32) words of 32 bits per lane in D / 32 / W blocks of 256 W bytes:
//   K  lane (g, r) = (lane / 16, lane % 16): word i holds channels 32 i + 8 g .. + 7 of token r, low nibble first: byte b converts
//      to the operand pair (2 b, 2 b + 1).
//   V  lane (q, c): word i holds channels 32 i + c (a) and 32 i + 16 + c (b) of tokens 4 q .. 4 q + 3, one byte per token, so that
//      tokens that arrive one by one never share a byte.  Nibbles from bit 0: a0 b0 b1 a1 a2 b2 b3 a3: shifted right by 4 its
//      bytes 0 and 2 are the pairs (b0, b1) and (b2, b3), and with the upper nibbles of the word shifted by 8 (a0, a1) and (a2, a3).
//   scales: K [tile][token][run], V [tile][q][run][token]: a lane finds what it multiplies with in one piece.
#ifndef AMS_KV_H_
#define AMS_KV_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ams.h"

namespace ams_kv {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 16;  // tokens of a tile
// Bits of the largest scale that ams_kv_write stores, 10912; it stores positive ones, so larger bits are a NaN or none of its own.  The
// codes' largest value, 6, times any finite scale above it is no fp16 value.
constexpr uint32_t kTopScale = 0x7154;

// Bytes of a block's planes.
struct Planes {
  int codes, scales, block;
};
constexpr Planes planes(int head_dim, int page_size, int scale_group) {
  const int codes = page_size * head_dim / 2, scales = page_size * (head_dim / scale_group) * 2;
  return {codes, scales, 2 * (codes + scales)};
}

// Division by a number that the host knows, of anything below 2^31.
struct Divisor {
  uint32_t by, mul, shift;
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};
inline Divisor divisor(uint32_t by) {
  uint32_t bits = 0;
  while (bits < 31 && (1u << bits) < by) bits++;
  return {by, (uint32_t)(((1ull << (31 + bits)) + by - 1) / by), 31 + bits};  // rounded up: off by less than n / 2^31 of a unit
}

// What every kernel of the cache is told of it.  Lengths, tables and row starts are the device's: a captured call follows them.
struct View {
  uint8_t* pages;
  const int32_t *table, *lens, *starts;  // starts may be null: one row per sequence
  int64_t table_stride, page_bytes;      // page_bytes: of a page's blocks of all heads
  int n_pages, table_width, batch, kv_heads, rows;
  int page_size, codes, scales, block;
  Divisor page_tiles, heads;  // heads: of the cache
};

__device__ __forceinline__ int lane_id() { return (int)(threadIdx.x & 63); }

// First row of sequence b (b <= batch); whatever the caller's numbers are it lies in [0, rows].
__device__ __forceinline__ int row_start(const View& v, int b) {
  if (!v.starts) return min(b, v.rows);
  return min(max(v.starts[b], 0), v.rows);
}
// Tokens of sequence b that the table has places for.
__device__ __forceinline__ int kv_len(const View& v, int b) { return (int)min((int64_t)max(v.lens[b], 0), (int64_t)v.table_width * v.page_size); }

// The block of tile `tile` (>= 0) of sequence b, or null where the table names no page of the pool; and where in it the tile is.
__device__ __forceinline__ uint8_t* block_of(const View& v, int b, int tile, int head, int* in_page) {
  const int page = (int)v.page_tiles.quotient((uint32_t)tile);
  *in_page = tile - page * (int)v.page_tiles.by;
  if (page >= v.table_width) return nullptr;
  const int number = v.table[b * v.table_stride + page];
  if (number < 0 || number >= v.n_pages) return nullptr;
  return v.pages + number * v.page_bytes + (int64_t)head * v.block;
}

// Which sequence a wavefront's item belongs to, where those of sequence b begin at first(b), ascending: the largest b with
// first(b) <= item.  64 sequences at a time.
template <typename First>
__device__ __forceinline__ int sequence_of(int batch, int item, First first) {
  int found = 0;
  for (int b = 1; b < batch; b += 64) {
    const int mine = b + lane_id();
    const int n = __builtin_popcountll(__ballot(mine < batch && first(mine) <= item));
    found += n;
    if (n < 64) break;
  }
  return found;
}

// The larger of two halves each, as unsigned numbers: of fp16 values that are not negative the larger one.
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  const us2 x = __builtin_bit_cast(us2, a), y = __builtin_bit_cast(us2, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

__device__ __forceinline__ uint32_t bits(h2 x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ h2 halves(uint32_t x) { return __builtin_bit_cast(h2, x); }

// Two e2m1 codes (byte BYTE of w) as fp16.
template <int BYTE>
__device__ __forceinline__ h2 two_codes(uint32_t w) {
  return __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, BYTE));
}
// Eight channels of K: a word's codes times their run's scale, each product rounded to fp16 (as ams_dequant rounds it).
__device__ __forceinline__ h8 restore_k(uint32_t w, h2 s) {
  const h2 a = two_codes<0>(w) * s, b = two_codes<1>(w) * s, c = two_codes<2>(w) * s, d = two_codes<3>(w) * s;
  return __builtin_bit_cast(h8, u4{bits(a), bits(b), bits(c), bits(d)});
}
// Four tokens of V's channels a (32 i + c) and b (32 i + 16 + c), with the scales of tokens 0, 1 and 2, 3.
__device__ __forceinline__ void restore_v(uint32_t w, uint32_t s01, uint32_t s23, u2* a, u2* b) {
  const uint32_t x = (w & 0x0F0F0F0Fu) | ((w >> 8) & 0xF0F0F0F0u), y = w >> 4;
  *a = u2{bits(two_codes<0>(x) * halves(s01)), bits(two_codes<2>(x) * halves(s23))};
  *b = u2{bits(two_codes<0>(y) * halves(s01)), bits(two_codes<2>(y) * halves(s23))};
}

// A lane's words of a tile's codes: W of them per block of 256 W bytes.
template <int D>
struct Lane {
  static constexpr int kWords = D / 32, W = kWords < 4 ? kWords : 4, kBlocks = kWords / W;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const uint8_t* tile, uint32_t lane) {
#pragma unroll
    for (int p = 0; p < kBlocks; p++) {
      const uint8_t* at = tile + (p * 256 * W + lane * 4u * W);
      if constexpr (W == 2) {
        const u2 x = *(const u2*)at;
        w[0] = x[0], w[1] = x[1];
      } else {
        const u4 x = *(const u4*)at;
        w[4 * p] = x[0], w[4 * p + 1] = x[1], w[4 * p + 2] = x[2], w[4 * p + 3] = x[3];
      }
    }
  }
};

// The same through a buffer: `at` is the wavefront's offset in it.
template <int D>
__device__ __forceinline__ void load_words(Lane<D>& x, __amdgpu_buffer_rsrc_t from, uint32_t lane, int at) {
  constexpr int W = Lane<D>::W;
#pragma unroll
  for (int p = 0; p < Lane<D>::kBlocks; p++) {
    if constexpr (W == 2) {
      const u2 w = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(from, lane * 8, at, 0));
      x.w[0] = w[0], x.w[1] = w[1];
    } else {
      const u4 w = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(from, lane * 16 + p * 1024, at, 0));
      x.w[4 * p] = w[0], x.w[4 * p + 1] = w[1], x.w[4 * p + 2] = w[2], x.w[4 * p + 3] = w[3];
    }
  }
}

// N scales that lie together, two to a word.
template <int N>
struct Scales {
  static constexpr int WORDS = (N + 1) / 2;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const uint8_t* at) {
    if constexpr (N == 1) {
      w[0] = *(const uint16_t*)at;
    } else if constexpr (WORDS % 4 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) {
        const u4 x = *(const u4*)(at + 4 * i);
        w[i] = x[0], w[i + 1] = x[1], w[i + 2] = x[2], w[i + 3] = x[3];
      }
    } else if constexpr (WORDS == 2) {
      const u2 x = *(const u2*)at;
      w[0] = x[0], w[1] = x[1];
    } else {
      static_assert(WORDS == 1, "1, 2, 4 or a multiple of 8 scales");
      w[0] = *(const uint32_t*)at;
    }
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, uint32_t offset, int at) {
    static_assert(N <= 8, "up to 16 bytes");
    if constexpr (N == 1) {
      w[0] = __builtin_amdgcn_raw_buffer_load_b16(from, offset, at, 0);
    } else if constexpr (N == 2) {
      w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, offset, at, 0);
    } else if constexpr (N == 4) {
      const u2 x = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(from, offset, at, 0));
      w[0] = x[0], w[1] = x[1];
    } else {
      const u4 x = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(from, offset, at, 0));
      w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
    }
  }
  // scale i twice
  __device__ __forceinline__ h2 twice(int i) const {
    const h2 x = halves(w[i / 2]);
    return i % 2 ? h2{x[1], x[1]} : h2{x[0], x[0]};
  }
};

// LDS that one wavefront's lanes exchange values through: written before, read after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int V>
struct Int {
  static constexpr int value = V;
};
// go(Int<head_dim>, Int<scale_group>) for the sizes that there are kernels for.
template <typename Go>
void dispatch(int head_dim, int scale_group, Go go) {
  switch (head_dim * 1000 + scale_group) {
    case 64032: return go(Int<64>(), Int<32>());
    case 64064: return go(Int<64>(), Int<64>());
    case 128032: return go(Int<128>(), Int<32>());
    case 128064: return go(Int<128>(), Int<64>());
    case 128128: return go(Int<128>(), Int<128>());
    case 256032: return go(Int<256>(), Int<32>());
    case 256064: return go(Int<256>(), Int<64>());
    case 256128: return go(Int<256>(), Int<128>());
  }
}

// Host: checks what the entry points share and fills in the view.
int make_view(const ams_kv_cache* c, int64_t rows, View* v);
bool aligned(const void* p, int bytes);
// AMS_OK on a gfx950 (ams_kernels.hip).
int device_status();
// Each file's kernels on the current device, so that a first call may be captured: one of a file brings in all of them.
inline bool loaded(const void* kernel) {
  hipFuncAttributes attributes;
  return hipFuncGetAttributes(&attributes, kernel) == hipSuccess;
}
bool load_cache();
bool load_stream();
bool load_tile();

}  // namespace ams_kv
#endif
