// Log probabilities behind the vocabulary projection: of given tokens, with their rank, the entropy and the most likely tokens.
//
//   x = logits / T,  lse = log sum exp x,  logprob = x[token] - lse,  entropy = lse - sum p x,  p = exp(x - lse)
//
// One read of the logits.  A wavefront walks pieces of a row with a running maximum m, S = sum 2^y and U = sum y 2^y, y = log2(e) / T (x - m):
// the log probability is ln 2 (y - log2 S) and the entropy ln 2 (log2 S - U / S), sums of terms of one sign.  m is always the true maximum of
// what has been seen, so neither difference cancels.  A wavefront's most likely tokens are a sorted list, one to a lane; what does not
// pass the last of them, which is nearly everything, costs one comparison of a lane's maximum.
//
// A row is shared out to several workgroups where rows do not fill the chip: each leaves its statistics and list in the workspace and
// counts itself in; the last one joins them, always in the same order, and clears the count.  Nobody waits for anybody.
#include <float.h>
#include <limits.h>

#include <algorithm>

#include "ams_kv_attention.h"

namespace ams_kv {

constexpr int kLogWaves = 4;
constexpr size_t kLogCountBytes = 64 * 1024;  // of a workspace: one count for each row, at its front
constexpr int kMaxRowParts = 64;

struct LogArgs {
  const void* logits;
  int64_t stride;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprobs;
  int32_t *rank, *top_tokens;
  uint32_t* counts;
  uint8_t* left;  // [row][part][LogStats, top entries]
  int vocab, top;
  float scale2;     // log2(e) / T
  int part_chunks;  // of a workgroup
  int part_bytes;
  uint32_t left_bytes;
  Divisor parts;
};

struct LogStats {
  float top, sum, moment;
  int ahead;
};

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
__device__ __forceinline__ float lane_value(float x, int lane) { return __builtin_bit_cast(float, of_lane(__builtin_bit_cast(int, x), lane)); }

// The n-th largest (from 0 on) of the lanes' values, none of them NaN: sorted by a bitonic network.
__device__ __forceinline__ float nth_of_lanes(float x, int n) {
  const int lane = lane_id();
#pragma unroll
  for (int k = 2; k <= 64; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2) {
      const float y = __shfl_xor(x, j, 64);
      x = ((lane & j) == 0) == ((lane & k) == 0) ? fmaxf(x, y) : fminf(x, y);
    }
  return lane_value(x, n);
}

// The wavefront's best entries, the n-th in lane n: by value, of equal ones the lower index first.  Lanes without one: -inf and no index.
struct TopList {
  float value = -INFINITY;
  int index = INT_MAX;
  float last_value = -INFINITY;  // of the last one that counts
  int last_index = INT_MAX;
  __device__ __forceinline__ bool full() const { return last_index != INT_MAX; }
  __device__ __forceinline__ bool takes(float v, int i) const { return v > last_value || (v == last_value && i < last_index); }
  __device__ __forceinline__ void insert(float v, int i, int top) {
    const int at = __builtin_popcountll(__ballot(value > v || (value == v && index < i)));
    const float up_value = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, value), 0x138, 0xF, 0xF, true));  // of the lane before
    const int up_index = __builtin_amdgcn_update_dpp(0, index, 0x138, 0xF, 0xF, true);
    const int lane = lane_id();
    value = lane > at ? up_value : lane == at ? v : value;
    index = lane > at ? up_index : lane == at ? i : index;
    last_value = lane_value(value, top - 1), last_index = of_lane(index, top - 1);
  }
  // The lanes' values that belong in the list.
  __device__ __forceinline__ void offer(float v, int i, float least, int top) {
    for (;;) {
      const unsigned long long some = __ballot(v >= least && i != INT_MAX && takes(v, i));
      if (!some) return;
      const int lane = __builtin_ctzll(some);
      insert(lane_value(v, lane), of_lane(i, lane), top);
      if (lane_id() == lane) i = INT_MAX;
    }
  }
};

// Pieces of 16 bytes of a row, kPieces to a lane; those of a lane are 64 pieces apart.
constexpr int kPieces = 4;
typedef u4 u4_unaligned __attribute__((aligned(2)));
template <typename T>
struct Chunk {
  static constexpr int PER = 16 / sizeof(T), VALUES = 64 * kPieces * PER;
  u4 raw[kPieces];
  __device__ __forceinline__ static int index(int first, int piece, int j) { return first + (piece * 64 + lane_id()) * PER + j; }
  __device__ __forceinline__ void load(const T* row, int first, int vocab) {
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
      const int at = index(first, u, 0);
      if (first + VALUES <= vocab || at + PER <= vocab) {
        raw[u] = *(const u4_unaligned*)(row + at);
      } else {
        T x __attribute__((ext_vector_type(PER)));
#pragma unroll
        for (int j = 0; j < PER; j++) {
          x[j] = -INFINITY;
          if (at + j < vocab) x[j] = row[at + j];
        }
        raw[u] = __builtin_bit_cast(u4, x);
      }
    }
  }
  __device__ __forceinline__ float value(int piece, int j) const {
    if constexpr (PER == 4) {
      return __builtin_bit_cast(f4, raw[piece])[j];
    } else {
      return (float)__builtin_bit_cast(h8, raw[piece])[j];
    }
  }
};

template <typename T>
__global__ __launch_bounds__(64 * kLogWaves) void logprobs_kernel(LogArgs a) {
  constexpr int PER = Chunk<T>::PER, VALUES = Chunk<T>::VALUES;
  const int wave = uniform((int)threadIdx.x >> 6), lane = lane_id();
  const uint32_t row = a.parts.quotient(blockIdx.x), part = blockIdx.x - row * a.parts.by;
  const T* const x = (const T*)a.logits + (int64_t)row * a.stride;
  __shared__ LogStats wave_stats[kLogWaves];
  __shared__ float list_values[kLogWaves][64];
  __shared__ int list_indexes[kLogWaves][64];
  __shared__ bool is_last;
  const int n_chunks = (a.vocab - 1) / VALUES + 1, end = min((int)(part + 1) * a.part_chunks, n_chunks);
  const int token = a.tokens ? a.tokens[row] : -1;
  const bool has_token = (uint32_t)token < (uint32_t)a.vocab;
  const float given = has_token ? (float)x[token] : 0;

  // x's scaled distance from m.  In 32 bits x may be as large as that type's values are: the difference first.
  auto scaled = [&](float v, float m) {
    if constexpr (PER == 4)
      return (v - m) * a.scale2;
    else
      return __builtin_fmaf(v, a.scale2, -(m * a.scale2));
  };
  // What m instead of `before` makes of it: for fp16 the difference of the products as they were rounded.
  auto moved = [&](float before, float m) {
#pragma clang fp contract(off)
    if constexpr (PER == 4) return (before - m) * a.scale2;
    const float from = before * a.scale2, to = m * a.scale2;
    return from - to;
  };
  float m = -INFINITY, sums[4] = {0, 0, 0, 0}, moments[4] = {0, 0, 0, 0};
  int ahead = 0;
  TopList list;
  int chunk = (int)part * a.part_chunks + wave;
  Chunk<T> now, next;
  if (chunk < end) now.load(x, chunk * VALUES, a.vocab);
  for (; chunk < end; chunk += kLogWaves) {
    const int first = chunk * VALUES;
    if (chunk + kLogWaves < end) next.load(x, (chunk + kLogWaves) * VALUES, a.vocab);
    float most[kPieces], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kPieces; u++) {
      most[u] = -INFINITY;
#pragma unroll
      for (int j = 0; j < PER; j++) most[u] = fmaxf(most[u], now.value(u, j));
      top = fmaxf(top, most[u]);
    }
    if (__ballot(top > m)) {
      const float before = m;
      m = max_over_wave(fmaxf(top, m));
      if (before != -INFINITY) {  // y becomes y + less
        const float less = moved(before, m), by = __builtin_amdgcn_exp2f(less);
#pragma unroll
        for (int i = 0; i < 4; i++) moments[i] = by > 0 ? by * __builtin_fmaf(less, sums[i], moments[i]) : 0.0f, sums[i] *= by;
      }
    }
    const float m_or_0 = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int u = 0; u < kPieces; u++)
#pragma unroll
      for (int j = 0; j < PER; j++) {
        const float y = scaled(now.value(u, j), m_or_0), e = __builtin_amdgcn_exp2f(y);
        sums[j & 3] += e;
        moments[j & 3] = __builtin_fmaf(e, fmaxf(y, -256.0f), moments[j & 3]);  // 2^y is 0 far above: so that 0 times an infinity is not asked for
      }
    if (has_token && __ballot(top >= given)) {
#pragma unroll
      for (int u = 0; u < kPieces; u++)
#pragma unroll
        for (int j = 0; j < PER; j++) {
          const float v = now.value(u, j);
          const int i = Chunk<T>::index(first, u, j);
          ahead += __builtin_popcountll(__ballot(i < a.vocab && (v > given || (v == given && i < token))));
        }
    }
    if (a.top > 0) {
      const unsigned long long some = __ballot(!list.full() || top > list.last_value);
      if (some) {
        // where many lanes have candidates most of them are not among the best: as many lanes' maxima as there are places say so
        const float least = __builtin_popcountll(some) > 6 ? nth_of_lanes(top, a.top - 1) : -INFINITY;
#pragma unroll
        for (int u = 0; u < kPieces; u++) {
          if (!__ballot(most[u] >= least && most[u] >= list.last_value)) continue;
#pragma unroll
          for (int j = 0; j < PER; j++) {
            const int i = Chunk<T>::index(first, u, j);
            list.offer(now.value(u, j), i < a.vocab ? i : INT_MAX, least, a.top);
          }
        }
      }
    }
    now = next;
  }

  // The workgroup's wavefronts, then the row's workgroups: wave 0 joins statistics and lists, in order.
  auto combine = [&](LogStats& s, LogStats t) {
    const float most = fmaxf(s.top, t.top);
    auto take = [&](const LogStats& p, float* sum, float* moment) {
      if (p.top == -INFINITY) return *sum = p.sum, *moment = p.moment, void();  // 0, unless something was a NaN
      const float less = moved(p.top, most), by = __builtin_amdgcn_exp2f(less);
      *moment = by > 0 || by != by ? by * __builtin_fmaf(less, p.sum, p.moment) : 0.0f, *sum = p.sum * by;
    };
    float sum[2], moment[2];
    take(s, &sum[0], &moment[0]), take(t, &sum[1], &moment[1]);
    s = {most, sum[0] + sum[1], moment[0] + moment[1], s.ahead + t.ahead};
  };
  LogStats mine = {m, sum_over_wave(sums[0] + sums[1] + (sums[2] + sums[3])), sum_over_wave(moments[0] + moments[1] + (moments[2] + moments[3])), ahead};
  auto join_waves = [&] {
    if (wave > 0) {
      if (lane == 0) wave_stats[wave] = mine;
      list_values[wave][lane] = list.value, list_indexes[wave][lane] = lane < a.top ? list.index : INT_MAX;
    }
    __syncthreads();
    if (wave == 0) {
      for (int w = 1; w < kLogWaves; w++) {
        combine(mine, wave_stats[w]);
        if (a.top > 0) list.offer(list_values[w][lane], list_indexes[w][lane], -INFINITY, a.top);
      }
    }
  };
  join_waves();

  if (a.parts.by > 1) {
    const __amdgpu_buffer_rsrc_t left = __builtin_amdgcn_make_buffer_rsrc((void*)a.left, 0, a.left_bytes, 0x00020000);
    const int first = (int)(row * a.parts.by) * a.part_bytes;
    if (wave == 0) {
      const int at = first + (int)part * a.part_bytes;
      if (lane == 0) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, mine), left, at, 0, kDeviceScope);
      if (lane < a.top) __builtin_amdgcn_raw_buffer_store_b64(u2{__builtin_bit_cast(uint32_t, list.value), (uint32_t)list.index}, left, at + 16 + 8 * lane, 0, kDeviceScope);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      is_last = __hip_atomic_fetch_add(a.counts + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts.by - 1;
      if (is_last) __hip_atomic_store(a.counts + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (!is_last) return;
    list = TopList();
    mine = {-INFINITY, 0, 0, 0};
    for (int p = wave; p < (int)a.parts.by; p += kLogWaves) {
      const int at = first + p * a.part_bytes;
      combine(mine, __builtin_bit_cast(LogStats, (u4)__builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(left, at, 0, kDeviceScope))));
      if (a.top > 0) {
        u2 entry = {0, INT_MAX};
        if (lane < a.top) entry = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(left, at + 16 + 8 * lane, 0, kDeviceScope));
        list.offer(__builtin_bit_cast(float, (uint32_t)entry[0]), (int)entry[1], -INFINITY, a.top);
      }
    }
    join_waves();
  }
  if (wave > 0) return;
  const float total = __log2f(mine.sum);
  auto log_probability = [&](float v) { return v == -INFINITY && mine.sum == mine.sum ? -INFINITY : (scaled(v, mine.top) - total) * 0.69314718056f; };
  if (lane == 0) {
    if (a.logprob) a.logprob[row] = has_token ? log_probability(given) : 0.0f;
    if (a.rank) a.rank[row] = has_token ? mine.ahead : -1;
    if (a.entropy) a.entropy[row] = mine.top == -INFINITY && mine.sum == 0 ? 0.0f : (total - mine.moment / mine.sum) * 0.69314718056f;
  }
  if (lane < a.top) {
    const bool there = list.index != INT_MAX;  // fewer tokens than places: none
    a.top_logprobs[(int64_t)row * a.top + lane] = there ? log_probability(list.value) : -INFINITY;
    a.top_tokens[(int64_t)row * a.top + lane] = there ? list.index : -1;
  }
}

bool load_logprobs() { return loaded((const void*)logprobs_kernel<float>); }

// Workgroups of a row.
struct LogPlan {
  int parts, part_chunks, part_bytes;
  size_t workspace;
};
static LogPlan log_plan(int type, int64_t rows, int64_t vocab, int top, size_t workspace) {
  const int64_t values = type == AMS_TYPE_FP32 ? Chunk<float>::VALUES : Chunk<_Float16>::VALUES;
  const int64_t chunks = std::max<int64_t>((vocab + values - 1) / values, 1);
  LogPlan p = {1, (int)chunks, 16 + 8 * top, 0};
  constexpr int64_t kWorkgroups = 1024;
  int64_t parts = std::min<int64_t>(std::min<int64_t>((chunks + kLogWaves - 1) / kLogWaves, kMaxRowParts), rows > 0 ? kWorkgroups / rows : 1);
  if (rows * (int64_t)sizeof(uint32_t) > (int64_t)kLogCountBytes) parts = 1;
  if (parts < 2) return p;
  p.part_chunks = (int)((chunks + parts - 1) / parts);
  p.parts = (int)((chunks + p.part_chunks - 1) / p.part_chunks);
  p.part_bytes = (p.part_bytes + 15) / 16 * 16;
  p.workspace = kLogCountBytes + (size_t)(rows * p.parts) * p.part_bytes;
  if (p.parts < 2 || workspace < p.workspace) return {1, (int)chunks, 16 + 8 * top, 0};
  return p;
}
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
  a.part_chunks = p.part_chunks, a.part_bytes = p.part_bytes, a.left_bytes = (uint32_t)(p.workspace ? p.workspace - kLogCountBytes : 0), a.parts = divisor((uint32_t)p.parts);
  const unsigned grid = (unsigned)(rows * p.parts);
  if (type == AMS_TYPE_FP32)
    hipLaunchKernelGGL(logprobs_kernel<float>, dim3(grid), dim3(64 * kLogWaves), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(logprobs_kernel<_Float16>, dim3(grid), dim3(64 * kLogWaves), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? AMS_OK : AMS_ERR_LAUNCH;
}

}  // extern "C"
