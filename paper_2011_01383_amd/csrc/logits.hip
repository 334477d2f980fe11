// The last layer's output made ready for the choice of the next token:
// penalties from the text so far, biases, the grammar's mask, the greedy token
// and the normaliser, in one pass over the logits.
//
// A workgroup takes one tile of one row's vocabulary: eight or sixteen logits a
// thread, loaded first.  While they are on their way it counts the row's history and
// biases that fall into the tile, in LDS with integer atomics (their order does
// not matter), and marks the touched places in a bitmap; the many that are not
// touched are only masked.  The bytes of the logits, in and out, would bound it:
// 256 rows of 131,072 bf16 logits take 23 us copied alone, 60 with histories of
// 1,024 to 2,048 tokens (17 of it), biases, masks and the normaliser (18: the
// reductions and a row's arrivals); one row of 32,000 takes 9.  The
// workgroup that ends a row last joins the tiles' maxima and sums, in tile
// order, so a call's result does not depend on which one that is.
#include "sequence.hpp"

namespace cortex {

constexpr int kSmallThreads = 256, kSmallTile = 2048, kLargeThreads = 1024, kLargeTile = 16384;
constexpr int kMaxBiases = 65535;                    // of a row
constexpr int kLogitsMaxRows = 65535;
constexpr size_t kLogitsCounterBytes = 256 * 1024;   // one arrival counter a row, at a fixed place for calls of every size

// One entry per logit of a tile: how often the row's own output holds it, and in
// the highest bit whether its prompt does.  16 bits while no history is longer
// than they count.
template <typename E> struct Counts {
  static constexpr uint32_t kSeen = 1u << (8 * sizeof(E) - 1);
  static constexpr int kPer = 4 / (int)sizeof(E);
  static __device__ __forceinline__ uint32_t *word(uint32_t *t, int i) { return t + i / kPer; }
  static __device__ __forceinline__ int shift(int i) { return i % kPer * 8 * (int)sizeof(E); }
  static __device__ __forceinline__ uint32_t get(const uint32_t *t, int i) { return ((const E *)t)[i]; }
};

struct LogitsPart {
  float top;       // the tile's largest value (NaN if it holds one)
  int32_t at;      // its index, -1 if every entry is -infinity
  float sum;       // sum of exp(v - top)
  float pad;
};

// Whether (v, i) comes before (w, j) as the row's choice: a NaN is the largest, equals go by index.
__device__ __forceinline__ bool chosen(float v, int i, float w, int j) {
  const bool vn = v != v, wn = w != w;
  if (vn != wn) return vn;
  if (vn || v == w) return i < j;
  return v > w;
}

// Joins two parts of a row.  Parts with nothing allowed have top = -infinity, sum = 0.
// Member by member: a choice between the structs would go through memory.
__device__ __forceinline__ LogitsPart join(const LogitsPart p, const LogitsPart q) {
  const bool first = q.at < 0 || (p.at >= 0 && chosen(p.top, p.at, q.top, q.at));
  const float top = first ? p.top : q.top;
  const float a = p.top == top ? 1.0f : fast_exp2((p.top - top) * kLog2e);
  const float b = q.top == top ? 1.0f : fast_exp2((q.top - top) * kLog2e);
  return LogitsPart{top, first ? p.at : q.at, p.sum * a + q.sum * b, 0.0f};
}

struct RowRules {
  float repetition, frequency, presence;
};

// Each operation rounded on its own, in the order the header gives.
__device__ __forceinline__ float apply_rules(float v, uint32_t n, const RowRules &r) {
#pragma clang fp contract(off)
  v = v > 0.0f ? v / r.repetition : v * r.repetition;
  const float f = r.frequency * (float)n;
  v = v - f;
  if (n) v = v - r.presence;
  return v;
}

__device__ __forceinline__ LogitsPart join_lanes(LogitsPart p, int lane) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const LogitsPart q = {__shfl_xor(p.top, s), __shfl_xor(p.at, s), __shfl_xor(p.sum, s), 0.0f};
    // both lanes of a pair add in the same order
    const bool upper = lane & s;
    const LogitsPart lo = {upper ? q.top : p.top, upper ? q.at : p.at, upper ? q.sum : p.sum, 0.0f};
    const LogitsPart hi = {upper ? p.top : q.top, upper ? p.at : q.at, upper ? p.sum : q.sum, 0.0f};
    p = join(lo, hi);
  }
  return p;
}

// Adds the values v[0..V) at index `at` and on to a part, one by one.
template <int V> __device__ void add_values(LogitsPart &part, const float (&v)[V], int at) {
#pragma unroll
  for (int k = 0; k < V; ++k)
    if (v[k] != -__builtin_inff()) part = join(part, LogitsPart{v[k], at + k, v[k] != v[k] ? v[k] : 1.0f, 0.0f});
}

template <typename T, typename E, int THREADS, int kTile, bool WIDE>
__global__ void __launch_bounds__(THREADS) logits_kernel(cortex_logits_t a, int32_t *status, uint32_t *counters,
                                                         LogitsPart *parts) {
  constexpr int V = 16 / (int)sizeof(T), NV = kTile / THREADS / V;
  typedef Counts<E> Count;
  typedef Counts<uint16_t> Entry;
  extern __shared__ uint32_t table[];            // [kTile] counts, then [kTile] of 16 bits: 1 + the entry of the row's biases
  __shared__ uint32_t touched[kTile / 32];
  __shared__ LogitsPart wave_part[THREADS / 64];
  __shared__ float wave_top[THREADS / 64], wave_sums[THREADS / 64];
  __shared__ int first_at;
  const int failed = entry_status(status);       // looked at, by all together, at the first barrier
  const int tid = (int)threadIdx.x, lane = tid & 63, row = (int)blockIdx.y, tiles = (int)gridDim.x;
  const int v0 = (int)blockIdx.x * kTile;
  const int width = a.vocab - v0 < kTile ? a.vocab - v0 : kTile;
  const T *src = (const T *)a.logits + (int64_t)row * a.logits_ld + v0;
  T *dst = a.out ? (T *)a.out + (int64_t)row * a.out_ld + v0 : nullptr;

  // V logits from i on; what is past the row's end repeats its last
  typedef T vec __attribute__((ext_vector_type(V)));
  vec raw[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = (j * THREADS + tid) * V;
    if (WIDE && i + V <= width) {
      raw[j] = *(const vec *)(src + i);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) raw[j][k] = src[i + k < width ? i + k : width - 1];
    }
  }

  int len = 0, prompt = 0, bias0 = 0, bias1 = 0, m = -1;
  bool broken = false;
  if (a.history_len) {
    len = a.history_len[row];
    prompt = a.prompt_len ? a.prompt_len[row] : 0;
    if (len < 0 || len > a.history_cap || prompt < 0 || prompt > len) broken = true;
  }
  if (a.bias_offsets) {
    bias0 = a.bias_offsets[row];
    bias1 = a.bias_offsets[row + 1];
    if (bias0 < 0 || bias1 < bias0 || bias1 > a.num_biases || bias1 - bias0 > kMaxBiases || (row == 0 && bias0 != 0) ||
        (row == a.rows - 1 && bias1 != a.num_biases))
      broken = true;
  }
  if (a.mask) {
    m = a.mask_index ? a.mask_index[row] : row;
    if (m < -1 || m >= a.mask_rows) broken = true;
  }
  if (broken) {
    if (tid == 0) raise_status(status, CORTEX_ST_INPUT_RANGE);
    return;
  }
  // the mask's words for the thread's values: V divides 32
  uint32_t open[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = (j * THREADS + tid) * V;
    open[j] = ~0u;
    if (m >= 0 && i < width) open[j] = a.mask[(int64_t)m * a.mask_ld + (v0 + i) / 32] >> (i % 32);
    if (i + V > width) open[j] &= i < width ? (1u << (width - i)) - 1u : 0u;
  }
  uint32_t *count = table, *bias = table + kTile / Count::kPer;
  const int words = kTile / Count::kPer + (a.bias_offsets ? kTile / Entry::kPer : 0);
  const u32x4 zeros = {0, 0, 0, 0};
  for (int k = tid * 4; k < words; k += THREADS * 4) *(u32x4 *)&table[k] = zeros;
  if (tid < kTile / 32) touched[tid] = 0;
  if (tid == 0) first_at = 0x7fffffff;
  // Another workgroup's error may be seen by some waves and not by others.  None goes
  // on alone: the tables' entries become places in bias_values.
  if (__syncthreads_or(failed != 0)) return;
  bool outside = false;
  const int32_t *text = a.history + (int64_t)row * a.history_ld;
#pragma unroll 4
  for (int j = tid; j < len; j += THREADS) {
    const int tok = text[j], i = tok - v0;
    outside |= tok < 0 || tok >= a.vocab;
    if (tok >= v0 && i < width) {
      atomicOr(&touched[i / 32], 1u << (i % 32));
      if (j < prompt) atomicOr(Count::word(count, i), Count::kSeen << Count::shift(i));
      else atomicAdd(Count::word(count, i), 1u << Count::shift(i));
    }
  }
  for (int j = bias0 + tid; j < bias1; j += THREADS) {
    const int tok = a.bias_tokens[j], i = tok - v0;
    outside |= tok < 0 || tok >= a.vocab;
    if (tok >= v0 && i < width) {
      atomicOr(&touched[i / 32], 1u << (i % 32));
      // the largest entry; another lane's change of the word starts it over
      const uint32_t entry = (uint32_t)(j - bias0) + 1u;
      uint32_t *w = Entry::word(bias, i), was = *w;
      while ((was >> Entry::shift(i) & 0xffffu) < entry) {
        const uint32_t found = atomicCAS(w, was, (was & ~(0xffffu << Entry::shift(i))) | entry << Entry::shift(i));
        if (found == was) break;
        was = found;
      }
    }
  }
  if (outside) raise_status(status, CORTEX_ST_INPUT_RANGE);
  __syncthreads();

  RowRules rules;
  rules.repetition = a.repetition ? a.repetition[row] : 1.0f;
  rules.frequency = a.frequency ? a.frequency[row] : 0.0f;
  rules.presence = a.presence ? a.presence[row] : 0.0f;
  // the values at i .. i + V - 1, -infinity past the row's end
  auto values = [&](int i, const vec &r, uint32_t allowed, float (&v)[V]) {
    const uint32_t changed = touched[i / 32] >> (i % 32) & ((1u << V) - 1u);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = to_float<T>(r[k]);
    if (changed)
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (changed >> k & 1) {
          const uint32_t c = Count::get(count, i + k), e = a.bias_offsets ? Entry::get(bias, i + k) : 0u;
          if (c) v[k] = apply_rules(v[k], c & ~Count::kSeen, rules);
          if (e) v[k] += a.bias_values[bias0 + (int)e - 1];
        }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const unsigned int keep = (unsigned int)((int)(allowed << (31 - k)) >> 31);
      v[k] = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned int, v[k]) & keep) | (0xff800000u & ~keep));
    }
  };

  // Largest value and the sum of exponentials below it.  fmax drops a NaN and
  // inf - inf makes one: a sum that is not a number sends the workgroup over its
  // values again, one by one.
  float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = (j * THREADS + tid) * V;
    if (i < width) {
      float v[V];
      values(i, raw[j], open[j], v);
      if (dst) {
        if (WIDE && i + V <= width) {
          Pack<T, V>::store(dst + i, v);
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (i + k < width) dst[i + k] = from_float<T>(v[k]);
        }
      }
      float high = v[0];
#pragma unroll
      for (int k = 1; k < V; ++k) high = __builtin_fmaxf(high, v[k]);
      const float old = top;
      top = __builtin_fmaxf(top, high);
      const float base = top == -__builtin_inff() ? 0.0f : top;
      sum *= fast_exp2((old - base) * kLog2e);
#pragma unroll
      for (int k = 0; k < V; ++k) sum += fast_exp2((v[k] - base) * kLog2e);
    }
  }
  if (!a.token && !a.lse) return;
  const float wtop = wave_max(top);
  if (lane == 0) wave_top[tid / 64] = wtop;
  LogitsPart part = {-__builtin_inff(), -1, 0.0f, 0.0f};
  if (__syncthreads_or(sum != sum)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = (j * THREADS + tid) * V;
      if (i < width) {
        float v[V];
        values(i, raw[j], open[j], v);
        add_values(part, v, v0 + i);
      }
    }
    part = join_lanes(part, lane);
    if (lane == 0) wave_part[tid / 64] = part;
    __syncthreads();
    if (tid >= 64) return;
    part = wave_part[lane % (THREADS / 64)];
    if (lane >= THREADS / 64) part = LogitsPart{-__builtin_inff(), -1, 0.0f, 0.0f};
    part = join_lanes(part, lane);
  } else {
    float high = wave_top[0];
#pragma unroll
    for (int k = 1; k < THREADS / 64; ++k) high = __builtin_fmaxf(high, wave_top[k]);
    const bool some = high > -__builtin_inff();
    const float all = wave_sum(some ? sum * fast_exp2((top - high) * kLog2e) : 0.0f);
    if (lane == 0) wave_sums[tid / 64] = all;
    if (some && top == high) {                   // few lanes: where it is
      int at = 0x7fffffff;
#pragma unroll
      for (int j = NV - 1; j >= 0; --j) {
        const int i = (j * THREADS + tid) * V;
        if (i < width) {
          float v[V];
          values(i, raw[j], open[j], v);
#pragma unroll
          for (int k = V - 1; k >= 0; --k)
            if (v[k] == high) at = v0 + i + k;
        }
      }
      atomicMin(&first_at, at);
    }
    __syncthreads();
    if (tid >= 64) return;
    float total = 0.0f;
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) total += wave_sums[k];
    if (some) part = LogitsPart{high, first_at, total, 0.0f};
  }
  if (tiles > 1) {
    unsigned int before = 0;
    if (lane == 0) {
      unsigned int *mine = (unsigned int *)(parts + (size_t)row * tiles + blockIdx.x);
      st_agent(mine, __builtin_bit_cast(unsigned int, part.top));
      st_agent(mine + 1, (unsigned int)part.at);
      st_agent(mine + 2, __builtin_bit_cast(unsigned int, part.sum));
      // The last of the row's workgroups finds the others' parts stored: they went past
      // the L2 (device scope), and are complete before the arrival.  A device-scope
      // fence would write back the whole L2, the row's output in it.
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      wave_stores_complete();
      before = __hip_atomic_fetch_add(counters + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (__builtin_amdgcn_readfirstlane(before) != (unsigned int)tiles - 1u) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    if (lane == 0) st_agent(counters + row, 0u);   // ready for the next call
    part = LogitsPart{-__builtin_inff(), -1, 0.0f, 0.0f};
    for (int t = 0; t < tiles; t += 64) {
      LogitsPart q = {-__builtin_inff(), -1, 0.0f, 0.0f};
      if (t + lane < tiles) {
        const unsigned int *p = (const unsigned int *)(parts + (size_t)row * tiles + t + lane);
        const unsigned int w0 = ld_agent(p), w1 = ld_agent(p + 1), w2 = ld_agent(p + 2);
        q = LogitsPart{__builtin_bit_cast(float, w0), (int32_t)w1, __builtin_bit_cast(float, w2), 0.0f};
      }
      part = join(part, join_lanes(q, lane));
    }
  }
  if (lane != 0) return;
  if (a.token) a.token[row] = part.at;
  if (a.lse) {
    float l = part.top;                          // -infinity, infinity or NaN as it is
    if (__builtin_fabsf(l) < __builtin_inff()) l += logf(part.sum);
    a.lse[row] = l;
  }
}

// Small tiles while the large ones would leave CUs without a workgroup.  The large
// ones count a row's history and end with an arrival eight times less often.
static bool small_tiles(int64_t rows, int64_t vocab) { return rows * ((vocab + kLargeTile - 1) / kLargeTile) < 256; }

template <typename T, typename E, int THREADS, int kTile>
int launch_logits_tiles(const cortex_logits_t &a, int32_t *status, void *ws, void *stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool wide = a.logits_ld % V == 0 && aligned16(a.logits) && (!a.out || (a.out_ld % V == 0 && aligned16(a.out)));
  const dim3 grid((a.vocab + kTile - 1) / kTile, a.rows);
  uint32_t *counters = (uint32_t *)ws;
  LogitsPart *parts = (LogitsPart *)((char *)ws + kLogitsCounterBytes);
  const size_t lds = kTile * (sizeof(E) + (a.bias_offsets ? sizeof(uint16_t) : 0));
  const void *kernel = wide ? (const void *)logits_kernel<T, E, THREADS, kTile, true>
                            : (const void *)logits_kernel<T, E, THREADS, kTile, false>;
  if (cached_occupancy(kernel, THREADS, lds) < 1) return CORTEX_E_HIP;   // also admits the LDS size
  if (wide) logits_kernel<T, E, THREADS, kTile, true><<<grid, THREADS, lds, (hipStream_t)stream>>>(a, status, counters, parts);
  else logits_kernel<T, E, THREADS, kTile, false><<<grid, THREADS, lds, (hipStream_t)stream>>>(a, status, counters, parts);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T, typename E> int launch_logits_counts(const cortex_logits_t &a, int32_t *status, void *ws, void *stream) {
  return small_tiles(a.rows, a.vocab) ? launch_logits_tiles<T, E, kSmallThreads, kSmallTile>(a, status, ws, stream)
                                      : launch_logits_tiles<T, E, kLargeThreads, kLargeTile>(a, status, ws, stream);
}

template <typename T> int launch_logits(const cortex_logits_t &a, int32_t *status, void *ws, void *stream) {
  return a.history_cap < 0x8000 ? launch_logits_counts<T, uint16_t>(a, status, ws, stream)
                                : launch_logits_counts<T, uint32_t>(a, status, ws, stream);
}

}  // namespace cortex

using namespace cortex;

extern "C" size_t cortex_logits_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || rows > kLogitsMaxRows || vocab < 1) return 0;
  return kLogitsCounterBytes + (size_t)rows * (((size_t)vocab + kSmallTile - 1) / kSmallTile) * sizeof(LogitsPart);
}

extern "C" int cortex_logits_process(const cortex_logits_t *args, int32_t *d_status, void *d_ws, size_t ws_bytes,
                                     void *stream) {
  if (!args || !d_status || !d_ws || !aligned16(d_ws)) return CORTEX_E_INVAL;
  const cortex_logits_t &a = *args;
  if ((a.dtype != CORTEX_F32 && a.dtype != CORTEX_BF16) || a.rows < 0 || a.rows > kLogitsMaxRows || a.vocab < 1 ||
      a.vocab > 0x7fff0000)
    return CORTEX_E_INVAL;
  if (!a.out && !a.token && !a.lse) return CORTEX_E_INVAL;
  if (a.logits_ld < a.vocab || (a.out && a.out_ld < a.vocab)) return CORTEX_E_INVAL;
  // an empty history has no address of its own
  if (a.history_cap < 0 || a.history_ld < a.history_cap || (a.history_cap > 0 && !a.history)) return CORTEX_E_INVAL;
  if (!a.history_len && (a.history || a.prompt_len || a.repetition || a.frequency || a.presence)) return CORTEX_E_INVAL;
  if (a.bias_offsets && (a.num_biases < 0 || (a.num_biases > 0 && (!a.bias_tokens || !a.bias_values)))) return CORTEX_E_INVAL;
  if (a.mask && (a.mask_rows < 0 || a.mask_ld < (a.vocab + 31) / 32 || (!a.mask_index && a.mask_rows < a.rows)))
    return CORTEX_E_INVAL;
  if (a.rows == 0) return CORTEX_OK;
  if (!a.logits) return CORTEX_E_INVAL;
  if (ws_bytes < cortex_logits_workspace_bytes(a.rows, a.vocab)) return CORTEX_E_WORKSPACE;
  return a.dtype == CORTEX_BF16 ? launch_logits<bf16_t>(a, d_status, d_ws, stream)
                                : launch_logits<float>(a, d_status, d_ws, stream);
}
