// Log probabilities behind the vocabulary projection: of given tokens, with their rank, the entropy and the most likely tokens.
//
//   x = logits / T,  lse = log sum exp x,  logprob = x[token] - lse,  entropy = lse - sum p x,  p = exp(x - lse)
//
// One read of the logits.  A wavefront walks pieces of a row with a running maximum m, S = sum 2^y and U = sum y 2^y, y = log2(e) / T (x - m):
// the log probability is ln 2 (y - log2 S) and the entropy ln 2 (log2 S - U / S), sums of terms of one sign.  m is always the true maximum of
// what has been seen, so neither difference cancels.
//
// The `top` most likely tokens.  The n-th largest of the maxima of disjoint pieces is a bound that n values reach, so nothing below it is among
// the n largest.  A wavefront takes that of the 256 pieces of its first chunk, by bisection, and writes down what reaches it: a few more
// than n values, from then on only larger ones.  (Where it has written down too much, it keeps the n largest and their last as the bound.)  At the
// end what reaches the largest bound of all wavefronts is counted out: a value's place is the number of those ahead of it.
//
// A row is shared out to several workgroups where rows do not fill the chip: each leaves its statistics and list in the workspace and
// counts itself in; the last one joins them, always in the same order, and clears the count.  Nobody waits for anybody.
//
// What bounds it.  Many rows: instruction issue beside memory: per value an exponential, four more operations and one for the rank, 9.7 with what
// is around them, 2048 rows of 128256 (525 MB) 92 us without tokens, 96 with, 102 with the most likely one, 126 with 20 (4.2 to 5.7 TB/s; a bare
// read takes 74).  Few rows: trips that follow one another: 1 row 5.6 us, with 5 tokens 10, with 20 13.9; of 32 rows with 20 (15 us) 1 is loading, 1.4 bisection, 1 writing down,
// 1.5 waiting for the other wavefronts, 2.5 joining their lists, 1.4 the way to memory and its count, 3.3 joining the parts.  Instructions
// that run once cost their way through the instruction cache: with 20 KB of code instead of 15 all that has a list took a third longer.
#include <float.h>
#include <limits.h>

#include <algorithm>

#include "ams_kv_attention.h"

namespace ams_kv {

constexpr size_t kLogCountBytes = 64 * 1024;  // of a workspace: one count for each row, at its front
constexpr int kMaxRowParts = 32;
constexpr int kWholeWaves = 4, kPartWaves = 8, kShortWaves = 16;  // of a workgroup that has a whole row of many, a part of one, or a short row
constexpr int kHeld = 256;  // values that a wavefront writes down at most

struct LogArgs {
  const void* logits;
  int64_t stride;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprobs;
  int32_t *rank, *top_tokens;
  uint32_t* counts;
  uint8_t* left;  // [row][part][LogStats, top entries]
  int vocab, top;
  float scale2;    // log2(e) / T
  int part_turns;  // of a workgroup: chunks of each of its wavefronts
  int part_bytes;
  uint32_t left_bytes;
  Divisor parts, by_top;
};

struct LogStats {
  float top, sum, moment;
  int ahead;
};
// A token and its logit in one number that is the larger the further ahead the token is: the value's bits in the order of the values (of
// both zeros the same), then the lower index.  0: none.
typedef uint64_t Entry;
__device__ __forceinline__ uint32_t key_of(float value) {
  const int bits = __builtin_bit_cast(int, value + 0.0f);
  return (uint32_t)(bits ^ (bits >> 31 | (int)0x80000000));
}
__device__ __forceinline__ Entry entry_of(float value, int index) { return (uint64_t)key_of(value) << 32 | ~(uint32_t)index; }
__device__ __forceinline__ float value_of(uint32_t key) { return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
__device__ __forceinline__ float value_of(Entry e) { return value_of((uint32_t)(e >> 32)); }
__device__ __forceinline__ int index_of(Entry e) { return (int)~(uint32_t)e; }
// How many of n entries are ahead of one; up to seven behind them are read, too.
template <int AT_ONCE>
__device__ __forceinline__ int place_of(const Entry* entries, int n, Entry mine) {
  int place = 0, i = 0;
  auto batch = [&](auto there) {
    Entry e[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++) e[j] = entries[i + j];
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++) place += (int)(e[j] > mine) & (int)there(j);
  };
#pragma unroll 1
  for (; i + AT_ONCE <= n; i += AT_ONCE) batch([](int) { return true; });
  if (i < n) batch([&](int j) { return i + j < n; });
  return place;
}

// Lanes' values joined over the wavefront, by lane patterns.
template <typename Join>
__device__ __forceinline__ float over_wave(float x, Join join) {
  auto from = [](float y, auto pattern) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, y), decltype(pattern)::value, 0xF, 0xF, true)); };
  x = join(x, from(x, Int<0xB1>()));   // lane ^ 1
  x = join(x, from(x, Int<0x4E>()));   // lane ^ 2
  x = join(x, from(x, Int<0x141>()));  // 7 - lane
  x = join(x, from(x, Int<0x140>()));  // 15 - lane
  const f2 y = with_16(x);
  x = join(y[0], y[1]);
  const f2 z = with_32(x);
  return join(z[0], z[1]);
}
__device__ __forceinline__ float max_over_wave(float x) {
  return over_wave(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_over_wave(float x) {
  return over_wave(x, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ int lanes_before(unsigned long long some) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0)); }

// Pieces of 16 bytes of a row, kPieces to a lane; those of a lane are 64 pieces apart.
constexpr int kPieces = 4;
typedef u4 u4_unaligned __attribute__((aligned(2)));
template <typename T>
struct Chunk {
  static constexpr int PER = 16 / sizeof(T), VALUES = 64 * kPieces * PER;
  u4 raw[kPieces];
  __device__ __forceinline__ static int index(int first, int piece, int j) { return first + (piece * 64 + lane_id()) * PER + j; }
  __device__ __forceinline__ void load(const T* row, int first, int vocab) {
    if (first + VALUES <= vocab) {
#pragma unroll
      for (int u = 0; u < kPieces; u++) raw[u] = *(const u4_unaligned*)(row + index(first, u, 0));
      return;
    }
    // The row's end: behind it -inf.  One piece may lie on it, for one lane in its middle.
    T edge __attribute__((ext_vector_type(PER)));
    const int whole = max(vocab - first, 0) / (64 * PER), at = index(first, whole, 0);
    u4 none;
#pragma unroll
    for (int j = 0; j < PER; j++) edge[j] = -INFINITY;
    none = __builtin_bit_cast(u4, edge);
    u4 last = none;
    if (at + PER <= vocab) {
      last = *(const u4_unaligned*)(row + at);
    } else if (at < vocab) {
#pragma unroll
      for (int j = 0; j < PER - 1; j++)
        if (at + j < vocab) edge[j] = row[at + j];
      last = __builtin_bit_cast(u4, edge);
    }
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
      raw[u] = u == whole ? last : none;
      if (u < whole) raw[u] = *(const u4_unaligned*)(row + index(first, u, 0));
    }
  }
  __device__ __forceinline__ T value(int piece, int j) const {
    typedef T Vector __attribute__((ext_vector_type(PER)));
    return __builtin_bit_cast(Vector, raw[piece])[j];
  }
  // The compiler is to convert the values again: kept from one use to the next they take 32 registers.
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int u = 0; u < kPieces; u++) asm volatile("" : "+v"(raw[u]));
  }
  // The largest of a piece; NaN is left out.
  __device__ __forceinline__ float largest(int piece) const {
    if constexpr (PER == 4) {
      const f4 x = __builtin_bit_cast(f4, raw[piece]);
      return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), -INFINITY);
    } else {
      const u4 r = raw[piece];
      const h2 x = __builtin_elementwise_max(__builtin_elementwise_max(halves(r[0]), halves(r[1])), __builtin_elementwise_max(halves(r[2]), halves(r[3])));
      return fmaxf(fmaxf((float)x[0], (float)x[1]), -INFINITY);
    }
  }
};

// The next smaller value of a type (of -inf and NaN themselves).
__device__ __forceinline__ float next_below(float x) {
  const int bits = __builtin_bit_cast(int, x);
  if (x == 0) return __builtin_bit_cast(float, 0x80000001u);
  return x > -INFINITY ? __builtin_bit_cast(float, bits < 0 ? bits + 1 : bits - 1) : x;
}
__device__ __forceinline__ _Float16 next_below(_Float16 x) {
  const short bits = __builtin_bit_cast(short, x);
  if (x == (_Float16)0) return __builtin_bit_cast(_Float16, (short)0x8001);
  return x > (_Float16)-INFINITY ? __builtin_bit_cast(_Float16, (short)(bits < 0 ? bits + 1 : bits - 1)) : x;
}

// A bound that n of the wavefront's 256 values reach and few others, -inf where fewer are above that; `most` is the largest of them.  Bisection
// of the bits in the order of the values, from the first in which they differ on, of 19 at most (all that fp16 values have), until no more
// than n reach it.
__device__ __forceinline__ float bound_of(const float (&x)[kPieces], float most, int n) {
  uint32_t keys[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; u++) keys[u] = key_of(x[u]);
  const uint32_t high = (uint32_t)uniform((int)key_of(most)), low = (uint32_t)uniform((int)key_of(-max_over_wave(-fminf(fminf(x[0], x[1]), fminf(x[2], x[3])))));
  const int first = high == low ? 0 : 31 - __builtin_clz(high ^ low);
  uint32_t key = high == low ? high : high & ~((2u << first) - 1);
#pragma unroll 1
  for (int bit = first; bit >= 13; bit--) {
    const uint32_t at = key | 1u << bit;
    int reach = 0;
#pragma unroll
    for (int u = 0; u < kPieces; u++) reach += __builtin_popcountll(__ballot(keys[u] >= at));
    if (reach >= n) key = at;
    if (reach == n) break;
  }
  return key < 0x00800000u ? -INFINITY : value_of(key);  // below: nothing but -inf
}

// What a wavefront has written down.
struct Held {
  Entry *entries, *spare;  // LDS, kHeld of them each
  int count = 0;
  float bound = -INFINITY;  // what is among the best is as large or larger; of later chunks larger
  Entry last = 0;           // and ahead of this one
  // Keeps the n first.  A place is the number of entries ahead.
  __device__ __forceinline__ void keep_best(int n) {
    wave_sync();
#pragma unroll 1
    for (int i = lane_id(); i < count; i += 64) {
      const Entry mine = entries[i];
      const int place = place_of<2>(entries, count, mine);
      if (place < n) spare[place] = mine;
    }
    wave_sync();
    count = min(count, n);
    if (lane_id() < count) entries[lane_id()] = spare[lane_id()];
    wave_sync();
    if (count == n) last = entries[n - 1], bound = value_of(last);
  }
  // Writes down the lanes' values in order of `bits`, each lane's lowest first.
  template <typename Value, typename Index>
  __device__ __forceinline__ void add(uint32_t bits, int n, float least, Value value, Index index) {
#pragma unroll 1
    while (__ballot(bits != 0)) {
      if (count + 64 > kHeld) keep_best(n);
      const int j = __builtin_ctz(bits | 0x80000000u);
      const float v = value(j);
      const Entry e = entry_of(v, index(j));
      const bool some = bits != 0 && v >= least && e > last;
      const unsigned long long lanes = __ballot(some);
      if (some) entries[count + lanes_before(lanes)] = e;
      count += __builtin_popcountll(lanes);
      bits &= bits - 1;
    }
  }
};

// Four wavefronts to a SIMD: six or eight make the compiler spill (2048 rows: 101, 105 and 277 us).
// COLD: the temperature is so low that products of fp16 logits with the factor may be 2^24 or more.
template <typename T, int WAVES, bool COLD>
__global__ __launch_bounds__(64 * WAVES, 4) void logprobs_kernel(LogArgs a) {
  constexpr int PER = Chunk<T>::PER, VALUES = Chunk<T>::VALUES, THREADS = 64 * WAVES;
  const int wave = uniform((int)threadIdx.x >> 6), lane = lane_id();
  const uint32_t row = a.parts.quotient(blockIdx.x), part = blockIdx.x - row * a.parts.by;
  const T* const x = (const T*)a.logits + (int64_t)row * a.stride;
  __shared__ __align__(16) Entry entries[2 * WAVES * kHeld + 8];  // of the wavefronts; those that are left of all
  __shared__ LogStats wave_stats[WAVES], row_stats;
  __shared__ float bounds[WAVES];
  __shared__ Entry best[64];
  __shared__ Entry least_entry;
  __shared__ int left_count;
  __shared__ bool is_last;
  if (threadIdx.x < 64) best[threadIdx.x] = 0;
  if (threadIdx.x < WAVES) bounds[threadIdx.x] = -INFINITY;
  if (threadIdx.x == 0) left_count = 0;
  __syncthreads();
  const int token = a.tokens ? a.tokens[row] : -1;
  const bool has_token = (uint32_t)token < (uint32_t)a.vocab;
  const T given = has_token ? x[token] : (T)0;
  const T below_given = next_below(given);
  const bool ranked = has_token && a.rank;

  // x's scaled distance from m.  In 32 bits x may be as large as that type's values are: the difference first.  In 16 it is one operation
  // with m's product, whose rounding moves all of a row's exponents alike, by half at most while that product is below 2^24.  Beyond, where the
  // nearest smaller value lies 2^12 away and only m itself has a weight, the factor's upper 13 bits do: their products with fp16 values are not
  // rounded.  (With this in all kernels a row of 20000 with 20 tokens took 10.7 us instead of 10.)
  static_assert(!COLD || PER == 8, "of 32 bits there is the difference");
  const float short_factor = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a.scale2) & 0xFFFFF800u);
  auto is_far = [&](float m) { return COLD && fabsf(m) * a.scale2 >= 16777216.0f; };
  auto factor_of = [&](float m) { return is_far(m) ? short_factor : a.scale2; };
  auto scaled = [&](float v, float m, float factor) {
    if constexpr (PER == 4)
      return (v - m) * a.scale2;
    else
      return __builtin_fmaf(v, factor, -(m * factor));
  };
  // What m instead of `before` makes of it: for fp16 the difference of the products as they were rounded.
  auto moved = [&](float before, float m) {
#pragma clang fp contract(off)
    if constexpr (PER == 4) return (before - m) * a.scale2;
    const float from = before * factor_of(before), to = m * factor_of(m);
    return from - to;
  };
  float factor = a.scale2;
  float m = -INFINITY, sums[4] = {0, 0, 0, 0}, moments[4] = {0, 0, 0, 0}, maxima[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; u++) maxima[u] = -INFINITY;
  int ahead = 0;
  int enough = 0;  // entries from which on a nearer bound is worth finding
  Held held = {entries + wave * kHeld, entries + (WAVES + wave) * kHeld};
  // A wavefront's chunks lie WAVES apart: a workgroup's form one window.
  const int begin = (int)part * a.part_turns * WAVES + wave, n_chunks = (a.vocab - 1) / VALUES + 1, end = min((int)(part + 1) * a.part_turns * WAVES, n_chunks);
  // Workgroups of whole rows ask for the next chunk as soon as there is one (2048 rows of 128256 108 -> 101 us); others have few (300 rows of 49999
  // in 32 bits 15.9 us, 19 with the registers for it).
  constexpr bool AHEAD = WAVES == kWholeWaves;
  Chunk<T> now, next;
  if (AHEAD && begin < end) now.load(x, begin * VALUES, a.vocab);
  for (int chunk = begin; chunk < end; chunk += WAVES) {
    const int first = chunk * VALUES;
    if (!AHEAD)
      now.load(x, first, a.vocab);
    else if (chunk + WAVES < end)
      next.load(x, first + WAVES * VALUES, a.vocab);
    float most[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; u++) most[u] = now.largest(u), maxima[u] = fmaxf(maxima[u], most[u]);
    const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    if (__ballot(top > m)) {
      const float before = m;
      m = max_over_wave(fmaxf(top, m));
      if constexpr (COLD) factor = factor_of(m);
      if (before != -INFINITY) {  // y becomes y + less
        const float less = moved(before, m), by = __builtin_amdgcn_exp2f(less);
#pragma unroll
        for (int i = 0; i < 4; i++) moments[i] = by > 0 ? by * __builtin_fmaf(less, sums[i], moments[i]) : 0.0f, sums[i] *= by;
      }
    }
    const float m_or_0 = m == -INFINITY ? 0.0f : m;
    now.forget();
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
      __builtin_amdgcn_sched_barrier(0);  // eight values at a time: more take registers
#pragma unroll
      for (int j = 0; j < PER; j++) {
        const float y = scaled((float)now.value(u, j), m_or_0, factor), e = __builtin_amdgcn_exp2f(y);
        sums[j & 3] += e;
        moments[j & 3] = __builtin_fmaf(e, fmaxf(y, -256.0f), moments[j & 3]);  // 2^y is 0 far above: so that 0 times an infinity is not asked for
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    now.forget();
    if (ranked && __ballot(top >= (float)given)) {
      // larger ones; of equal logits those that come before the token
      const T above = first + VALUES <= token ? below_given : given;
#pragma unroll
      for (int u = 0; u < kPieces; u++)
#pragma unroll
        for (int j = 0; j < PER; j++) ahead += __builtin_popcountll(__ballot(now.value(u, j) > above));
      if (first <= token && (token < first + VALUES || given == (T)-INFINITY)) {  // nothing is below -inf
        const int before = token - first - hidden(lane) * PER;  // values of the lane's first piece that come before it
#pragma unroll
        for (int u = 0; u < kPieces; u++)
#pragma unroll
          for (int j = 0; j < PER; j++) ahead += __builtin_popcountll(__ballot(now.value(u, j) == given && j < before - u * 64 * PER));
      }
    }
    now.forget();
    float least = -INFINITY;
    if (a.top > 0) {  // what the other wavefronts know: n values of theirs reach it
#pragma unroll
      for (int w = 0; w < WAVES; w++) least = fmaxf(least, __hip_atomic_load(&bounds[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
    }
    if (a.top > 0 && __ballot(top > held.bound && top >= least)) {
      // the first chunk, much that passes the bound or much written down since: a better one, of all that has been seen
      float own = -INFINITY;
      if (chunk == begin || held.count >= enough || __builtin_popcountll(__ballot(top > held.bound && top >= least)) > 24) {
        own = a.top == 1 ? m : bound_of(maxima, m, a.top);
        least = fmaxf(least, own);
        enough = held.count + max(a.top, 16);
      }
      const float from = fmaxf(fmaxf(least, held.bound), -FLT_MAX);  // never -inf
      uint32_t pieces = 0;  // of the lane; it takes one after the other, all lanes at once
#pragma unroll
      for (int u = 0; u < kPieces; u++) pieces |= most[u] >= from ? 1u << u : 0u;
#pragma unroll 1
      for (; __ballot(pieces != 0); pieces &= pieces - 1) {
        const int u = __builtin_ctz(pieces | 1u << kPieces);
        Chunk<T> piece;  // that one in place 0
        piece.raw[0] = now.raw[0];
#pragma unroll
        for (int i = 1; i < kPieces; i++) piece.raw[0] = u == i ? now.raw[i] : piece.raw[0];
        uint32_t some = 0;
#pragma unroll
        for (int j = 0; j < PER; j++) some |= (float)piece.value(0, j) >= from ? 1u << j : 0u;
        held.add(pieces ? some : 0, a.top, least, [&](int j) {
          T v = piece.value(0, 0);
#pragma unroll
          for (int i = 1; i < PER; i++) v = j == i ? piece.value(0, i) : v;
          return (float)v;
        }, [&](int j) { return Chunk<T>::index(first, u, j); });
      }
      if (own > held.bound) held.bound = own, held.last = entry_of(own, 0);  // equal ones that come later are not
      if (lane == 0) __hip_atomic_store(&bounds[wave], held.bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    if (AHEAD) now = next;
  }

  // Statistics of the workgroup's wavefronts, then of the row's workgroups, one to a lane: all of them for the largest maximum.
  auto joined = [&](const LogStats& s) {
    const float most = max_over_wave(s.top);
    float sum = s.sum, moment = s.moment;
    if (s.top != -INFINITY) {  // else 0, unless something was a NaN
      const float less = moved(s.top, most), by = __builtin_amdgcn_exp2f(less);
      moment = by > 0 ? by * __builtin_fmaf(less, sum, moment) : 0.0f, sum *= by;
    }
    return LogStats{most, sum_over_wave(sum), sum_over_wave(moment), (int)wave_sum((uint32_t)s.ahead)};
  };
  // What is left of several lists goes to `left`, and from there to its place.
  Entry* const left = entries + WAVES * kHeld;
  auto leave = [&](bool some, Entry e) {
    const unsigned long long lanes = __ballot(some);
    int at = 0;
    if (lane == 0 && lanes) at = atomicAdd(&left_count, __builtin_popcountll(lanes));
    at = uniform(at);
    if (some) left[at + lanes_before(lanes)] = e;
  };
  auto count_out = [&] {
    __syncthreads();
    const int n = left_count;
    for (int i = threadIdx.x; i < n; i += THREADS) {
      const Entry e = left[i];
      const int place = place_of<8>(left, n, e);
      if (place < a.top) best[place] = e;
    }
    __syncthreads();
  };
  const LogStats no_stats = {-INFINITY, 0, 0, 0};
  LogStats mine = {m, sum_over_wave(sums[0] + sums[1] + (sums[2] + sums[3])), sum_over_wave(moments[0] + moments[1] + (moments[2] + moments[3])), ahead};
  if (lane == 0) wave_stats[wave] = mine;
  __syncthreads();
  // wave 0 joins the statistics; where lists are joined too the last one does so meanwhile
  const int joins = a.top > 0 ? WAVES - 1 : 0;
  if (wave == joins) {
    mine = joined(lane < WAVES ? wave_stats[lane] : no_stats);
    if (lane == 0) row_stats = mine;
  }
  if (a.top > 0) {
    float bound = bounds[0];
#pragma unroll
    for (int w = 1; w < WAVES; w++) bound = fmaxf(bound, bounds[w]);
    for (int i0 = 0; i0 < held.count; i0 += 64) {
      const Entry e = held.entries[min(i0 + lane, held.count - 1)];
      leave(i0 + lane < held.count && value_of(e) >= bound, e);
    }
    count_out();
  }
  if (a.top > 0) mine = row_stats;

  if (a.parts.by > 1) {
    const __amdgpu_buffer_rsrc_t share = __builtin_amdgcn_make_buffer_rsrc((void*)a.left, 0, a.left_bytes, 0x00020000);
    const int first = (int)(row * a.parts.by) * a.part_bytes;
    if (wave == 0) {
      const int at = first + (int)part * a.part_bytes;
      if (lane == 0) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, mine), share, at, 0, kDeviceScope);
      if (lane < a.top) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, (Entry)best[lane]), share, at + 16 + 8 * lane, 0, kDeviceScope);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      is_last = __hip_atomic_fetch_add(a.counts + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts.by - 1;
      if (is_last) __hip_atomic_store(a.counts + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      left_count = 0, least_entry = 0;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (!is_last) return;
    // what reaches the last of a whole list of some part
    if (threadIdx.x < 64) best[threadIdx.x] = 0;
    const int n = (int)a.parts.by * a.top;
    Entry theirs_best[kMaxRowParts * AMS_LOGPROBS_MAX_TOP / THREADS], bound = 0;
#pragma unroll
    for (int k = 0; k < kMaxRowParts * AMS_LOGPROBS_MAX_TOP / THREADS; k++) {
      const int i = k * THREADS + (int)threadIdx.x, p = (int)a.by_top.quotient((uint32_t)i);
      theirs_best[k] = 0;
      if (k * THREADS < n) theirs_best[k] = __builtin_bit_cast(Entry, __builtin_amdgcn_raw_buffer_load_b64(share, i < n ? first + p * a.part_bytes + 16 + 8 * (i - p * a.top) : 0x7FFE0000, 0, kDeviceScope));
    }
    LogStats theirs = no_stats;  // of the parts
    if (wave == joins && lane < (int)a.parts.by) theirs = __builtin_bit_cast(LogStats, (u4)__builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(share, first + lane * a.part_bytes, 0, kDeviceScope)));
    if (wave == joins) {
      mine = joined(theirs);
      if (lane == 0) row_stats = mine;
    }
    if (a.top > 0) {
      if (n > 256) __syncthreads();
#pragma unroll
      for (int k = 0; k < kMaxRowParts * AMS_LOGPROBS_MAX_TOP / THREADS; k++) {
        const int i = k * THREADS + (int)threadIdx.x;
        if (n > 256 && i < n && (i + 1) % a.top == 0 && theirs_best[k]) atomicMax((unsigned long long*)&least_entry, (unsigned long long)theirs_best[k]);
      }
      if (n > 256) {
        __syncthreads();
        bound = least_entry;
      }
#pragma unroll
      for (int k = 0; k < kMaxRowParts * AMS_LOGPROBS_MAX_TOP / THREADS; k++)
        if (k * THREADS < n) leave(theirs_best[k] != 0 && theirs_best[k] >= bound, theirs_best[k]);
      count_out();
      mine = row_stats;
    }
  }
  if (wave > 0) return;
  const float total = __log2f(mine.sum);
  auto log_probability = [&](float v) {
    const float y = is_far(mine.top) ? (v - mine.top) * a.scale2 : scaled(v, mine.top, a.scale2);
    return v == -INFINITY && mine.sum == mine.sum ? -INFINITY : (y - total) * 0.69314718056f;
  };
  if (lane == 0) {
    if (a.logprob) a.logprob[row] = has_token ? log_probability((float)given) : 0.0f;
    if (a.rank) a.rank[row] = has_token ? mine.ahead : -1;
    if (a.entropy) a.entropy[row] = mine.top == -INFINITY && mine.sum == 0 ? 0.0f : (total - mine.moment / mine.sum) * 0.69314718056f;
  }
  if (a.top == 0) return;
  // Fewer logits above -inf than places: then the first tokens with -inf; behind them none.
  const int found = min(__builtin_popcountll(__ballot(best[lane] != 0)), a.top);
  int filled = found;
  for (int i0 = 0; i0 < a.vocab && filled < a.top; i0 += 64) {
    const unsigned long long some = __ballot(i0 + lane < a.vocab && (float)x[min(i0 + lane, a.vocab - 1)] == -INFINITY);
    const int place = filled + lanes_before(some);
    if ((some >> lane & 1) && place < a.top) best[place] = entry_of(-INFINITY, i0 + lane);
    filled += __builtin_popcountll(some);
  }
  wave_sync();
  if (lane < a.top) {
    const Entry e = best[lane];
    a.top_logprobs[(int64_t)row * a.top + lane] = e ? log_probability(value_of(e)) : -INFINITY;
    a.top_tokens[(int64_t)row * a.top + lane] = e ? index_of(e) : -1;
  }
}

bool load_logprobs() { return loaded((const void*)logprobs_kernel<float, 8, false>); }

// Workgroups of a row.  Eight wavefronts to a workgroup up to as many as the chip holds at once, beyond that four, whose ends others cover (rows
// of 50001, 8 tokens: 300 rows 20.5 us with eight, 23 with four; 500 22.4 and 24.3; 600 32 and 29; 2048 74 and 61).  Where sixteen have a chunk of the
// row each, as of 32000 tokens in fp16, and every workgroup has a compute unit, they take it whole (rows of 20000 with 20 tokens: 1 row in two
// parts 11.7 us, whole 9.8; 128 rows 13.8 and 12.3; 200 rows with eight 13.3, sixteen 12.8; 300 rows 16.4 and 21.6).
constexpr int64_t kWorkgroups = 512;
struct LogPlan {
  int waves, parts, part_turns, part_bytes;
  size_t workspace;
};
static LogPlan log_plan(int type, int64_t rows, int64_t vocab, int top, size_t workspace) {
  const int64_t values = type == AMS_TYPE_FP32 ? Chunk<float>::VALUES : Chunk<_Float16>::VALUES, chunks = (vocab + values - 1) / values;
  const bool is_short = chunks > kPartWaves && chunks <= kShortWaves && rows <= 256;
  const int waves = rows > kWorkgroups ? kWholeWaves : is_short ? kShortWaves : kPartWaves;
  const LogPlan whole = {waves, 1, (int)((chunks + waves - 1) / waves), 0, 0};
  const int64_t turns = (chunks + kPartWaves - 1) / kPartWaves;
  const int64_t parts = std::min<int64_t>(std::min<int64_t>(turns, kMaxRowParts), rows > 0 ? kWorkgroups / rows : 1);
  // More than half as many rows as compute units: two parts have to be long to pay for their join (256 rows, 20 tokens, whole and in two: of 20000
  // 13.7 us and 16.8, 50001 19.4 and 22.9, 128256 33.5 and 32.1; 128 rows of 50001 19.0, in four 17.2).
  if (parts < 2 || is_short || (rows > 128 && turns < 4 * parts)) return whole;
  LogPlan p = {kPartWaves, 0, (int)((turns + parts - 1) / parts), (16 + 8 * top + 15) / 16 * 16, 0};
  p.parts = (int)((turns + p.part_turns - 1) / p.part_turns);
  p.workspace = kLogCountBytes + (size_t)(rows * p.parts) * p.part_bytes;
  return workspace < p.workspace ? whole : p;
}
static_assert(512 * sizeof(uint32_t) <= kLogCountBytes, "a count for each row that is shared out");
static_assert(kMaxRowParts * AMS_LOGPROBS_MAX_TOP <= kPartWaves * kHeld, "the parts' lists fit in LDS");
static bool log_sizes_ok(int type, int64_t rows, int64_t vocab, int top) {
  return (type == AMS_TYPE_FP16 || type == AMS_TYPE_FP32) && rows >= 0 && rows <= AMS_KV_MAX_TOKENS && vocab >= 1 && vocab <= AMS_LOGPROBS_MAX_VOCAB && top >= 0 && top <= AMS_LOGPROBS_MAX_TOP;
}

}  // namespace ams_kv

using namespace ams_kv;

extern "C" {

int ams_logprobs_workspace_bytes(int type, int64_t rows, int64_t vocab, int top, size_t* bytes) {
  if (!bytes) return AMS_ERR_NULL;
  if (!log_sizes_ok(type, rows, vocab, top)) return AMS_ERR_SHAPE;
  *bytes = log_plan(type, rows, vocab, top, SIZE_MAX).workspace;
  return AMS_OK;
}

int ams_logprobs(const void* logits, int type, int64_t rows, int64_t vocab, int64_t stride, const int32_t* tokens, float temperature, int top, float* logprob, int32_t* rank, float* entropy,
                 float* top_logprobs, int32_t* top_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  if (!log_sizes_ok(type, rows, vocab, top) || !(temperature >= 1e-6f) || !(temperature <= 1e6f)) return AMS_ERR_SHAPE;
  if (rows > 0 && (!logits || ((logprob || rank) && !tokens) || (top > 0 && (!top_logprobs || !top_tokens)))) return AMS_ERR_NULL;
  if (!aligned(logits, type == AMS_TYPE_FP32 ? 4 : 2) || !aligned(tokens, 4) || !aligned(logprob, 4) || !aligned(rank, 4) || !aligned(entropy, 4) || !aligned(top_logprobs, 4) || !aligned(top_tokens, 4) ||
      !aligned(workspace, 16))
    return AMS_ERR_ALIGN;
  if (const int rc = device_status(); rc != AMS_OK) return rc;
  if (rows == 0) return AMS_OK;
  const LogPlan p = log_plan(type, rows, vocab, top, workspace ? workspace_bytes : 0);
  LogArgs a = {};
  a.logits = logits, a.stride = stride, a.tokens = tokens, a.logprob = logprob, a.entropy = entropy, a.rank = rank, a.top_logprobs = top_logprobs, a.top_tokens = top_tokens;
  a.counts = (uint32_t*)workspace, a.left = (uint8_t*)workspace + kLogCountBytes;
  a.vocab = (int)vocab, a.top = top, a.scale2 = (float)(1.4426950408889634 / temperature);
  a.part_turns = p.part_turns, a.part_bytes = p.part_bytes, a.left_bytes = (uint32_t)(p.workspace ? p.workspace - kLogCountBytes : 0), a.parts = divisor((uint32_t)p.parts), a.by_top = divisor((uint32_t)std::max(top, 1));
  // One launch has fewer than 2^32 threads (of more the runtime leaves out what passes that, with no error).
  constexpr int64_t kLaunchRows = 1 << 23;  // of a workgroup each
  static_assert(kLaunchRows >= kWorkgroups && kLaunchRows * 64 * kWholeWaves < (int64_t)1 << 32, "rows that are shared out are one launch's");
  auto launch = [&](auto kernel) {
    for (int64_t left = rows;;) {
      const int64_t n = std::min(left, kLaunchRows);
      hipLaunchKernelGGL(kernel, dim3((unsigned)(n * p.parts)), dim3(64 * p.waves), 0, (hipStream_t)stream, a);
      if ((left -= n) == 0) return;
      a.logits = (const uint8_t*)a.logits + n * stride * (type == AMS_TYPE_FP32 ? 4 : 2);
      for (auto* t : {&a.logprob, &a.entropy})
        if (*t) *t += n;
      if (a.tokens) a.tokens += n;
      if (a.rank) a.rank += n;
      if (top > 0) a.top_logprobs += n * top, a.top_tokens += n * top;
    }
  };
  auto of_type = [&](auto zero, auto cold) {
    typedef decltype(zero) T;
    constexpr bool COLD = decltype(cold)::value != 0;
    if (p.waves == kWholeWaves) return launch(logprobs_kernel<T, kWholeWaves, COLD>);
    if (p.waves == kShortWaves) return launch(logprobs_kernel<T, kShortWaves, COLD>);
    launch(logprobs_kernel<T, kPartWaves, COLD>);
  };
  if (type == AMS_TYPE_FP32)
    of_type(0.0f, Int<0>());
  else if (65504 * a.scale2 < 16777216.0f)  // the largest fp16 value; temperatures above 0.0056
    of_type((_Float16)0, Int<0>());
  else
    of_type((_Float16)0, Int<1>());
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

}  // extern "C"
