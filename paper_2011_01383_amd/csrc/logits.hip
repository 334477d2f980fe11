// The last layer's output made ready for the choice of the next token:
// penalties from the text so far, biases, the grammar's mask, the greedy token
// and the normaliser, in one pass over the logits.
//
// A workgroup takes one tile of one row's vocabulary.  It first counts the
// row's history and biases that fall into the tile, in LDS with integer
// atomics (their order does not matter), then reads each logit once.  The
// workgroup that ends a row last joins the tiles' maxima and sums, in tile
// order, so a call's result does not depend on which one that is.
#include "sequence.hpp"

namespace cortex {

constexpr int kLogitsThreads = 256;
constexpr int kLogitsTile = 4096;
constexpr int kLogitsMaxRows = 65535;
constexpr size_t kLogitsCounterBytes = 256 * 1024;   // one arrival counter a row, at a fixed place for calls of every size
constexpr uint32_t kSeen = 0x80000000u;              // in the prompt; the bits below count the row's own output

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
__device__ __forceinline__ LogitsPart join(const LogitsPart &p, const LogitsPart &q) {
  LogitsPart r = chosen(p.top, p.at, q.top, q.at) ? p : q;
  if (p.at < 0) r = q;
  if (q.at < 0) r = p;
  if (p.at < 0 || q.at < 0) return r;
  const float a = p.top == r.top ? 1.0f : fast_exp2((p.top - r.top) * kLog2e);
  const float b = q.top == r.top ? 1.0f : fast_exp2((q.top - r.top) * kLog2e);
  r.sum = p.sum * a + q.sum * b;
  return r;
}

struct RowRules {
  float repetition, frequency, presence;
};

// Each operation rounded on its own, in the order the header gives.
__device__ __forceinline__ float apply_rules(float v, uint32_t count, const RowRules &r) {
#pragma clang fp contract(off)
  v = v > 0.0f ? v / r.repetition : v * r.repetition;
  const uint32_t n = count & ~kSeen;
  const float f = r.frequency * (float)n;
  v = v - f;
  if (n) v = v - r.presence;
  return v;
}

template <typename T, int V>
__global__ void __launch_bounds__(kLogitsThreads) logits_kernel(cortex_logits_t a, int32_t *status, uint32_t *counters,
                                                                LogitsPart *parts) {
  __shared__ uint32_t count[kLogitsTile];
  __shared__ uint32_t bias[kLogitsTile];      // 1 + the entry of the row's biases
  __shared__ LogitsPart wave_part[kLogitsThreads / 64];
  if (load_status(status) != 0) return;
  const int tid = (int)threadIdx.x, row = (int)blockIdx.y, tiles = (int)gridDim.x;
  const int v0 = (int)blockIdx.x * kLogitsTile;
  const int width = a.vocab - v0 < kLogitsTile ? a.vocab - v0 : kLogitsTile;

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
    if (bias0 < 0 || bias1 < bias0 || bias1 > a.num_biases || (row == 0 && bias0 != 0) ||
        (row == a.rows - 1 && bias1 != a.num_biases))
      broken = true;
  }
  if (a.mask || a.mask_index) {
    m = a.mask_index ? a.mask_index[row] : row;
    if (m < -1 || m >= a.mask_rows) broken = true;
  }
  if (broken) {
    if (tid == 0) raise_status(status, CORTEX_ST_INPUT_RANGE);
    return;
  }
  for (int i = tid; i < width; i += kLogitsThreads) count[i] = bias[i] = 0;
  __syncthreads();
  bool outside = false;
  for (int j = tid; j < len; j += kLogitsThreads) {
    const int tok = a.history[(int64_t)row * a.history_ld + j];
    outside |= tok < 0 || tok >= a.vocab;
    const int i = tok - v0;
    if (tok >= v0 && i < width) {
      if (j < prompt) atomicOr(&count[i], kSeen);
      else atomicAdd(&count[i], 1u);
    }
  }
  for (int j = bias0 + tid; j < bias1; j += kLogitsThreads) {
    const int tok = a.bias_tokens[j];
    outside |= tok < 0 || tok >= a.vocab;
    const int i = tok - v0;
    if (tok >= v0 && i < width) atomicMax(&bias[i], (uint32_t)(j - bias0) + 1u);
  }
  if (outside) raise_status(status, CORTEX_ST_INPUT_RANGE);
  __syncthreads();

  RowRules rules;
  rules.repetition = a.repetition ? a.repetition[row] : 1.0f;
  rules.frequency = a.frequency ? a.frequency[row] : 0.0f;
  rules.presence = a.presence ? a.presence[row] : 0.0f;
  const T *src = (const T *)a.logits + (int64_t)row * a.logits_ld + v0;
  T *dst = a.out ? (T *)a.out + (int64_t)row * a.out_ld + v0 : nullptr;
  const uint32_t *mask = m >= 0 ? a.mask + (int64_t)m * a.mask_ld + v0 / 32 : nullptr;

  LogitsPart part = {-__builtin_inff(), -1, 0.0f, 0.0f};
  for (int i = tid * V; i < width; i += kLogitsThreads * V) {
    const int n = width - i < V ? width - i : V;
    float v[V];
    if (n == V) Pack<T, V>::load(src + i, v);
    else
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = k < n ? to_float<T>(src[i + k]) : 0.0f;
    const uint32_t allowed = mask ? mask[i / 32] >> (i % 32) : ~0u;
    float top = -__builtin_inff();
    int at = -1;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (k < n) {
        const uint32_t c = count[i + k], b = bias[i + k];
        if (c) v[k] = apply_rules(v[k], c, rules);
        if (b) v[k] += a.bias_values[bias0 + (int)b - 1];
      }
      if (k >= n || !(allowed >> k & 1)) v[k] = -__builtin_inff();
      if (v[k] != -__builtin_inff() && (at < 0 || chosen(v[k], v0 + i + k, top, at))) {
        top = v[k];
        at = v0 + i + k;
      }
    }
    if (dst) {
      if (n == V) Pack<T, V>::store(dst + i, v);
      else
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (k < n) dst[i + k] = from_float<T>(v[k]);
    }
    if (at >= 0) {
      LogitsPart q = {top, at, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < V; ++k) q.sum += v[k] == top ? 1.0f : fast_exp2((v[k] - top) * kLog2e);
      part = join(part, q);
    }
  }
  auto from_lane = [](const LogitsPart &p, int mask_) {
    return LogitsPart{__shfl_xor(p.top, mask_), __shfl_xor(p.at, mask_), __shfl_xor(p.sum, mask_), 0.0f};
  };
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const LogitsPart q = from_lane(part, s);
    // both lanes of a pair add in the same order
    part = (tid & s) ? join(q, part) : join(part, q);
  }
  if ((tid & 63) == 0) wave_part[tid / 64] = part;
  __syncthreads();
  if (tid != 0 || (!a.token && !a.lse)) return;
  part = wave_part[0];
  for (int w = 1; w < kLogitsThreads / 64; ++w) part = join(part, wave_part[w]);
  if (tiles > 1) {
    unsigned int *mine = (unsigned int *)(parts + (size_t)row * tiles + blockIdx.x);
    st_agent(mine, __builtin_bit_cast(unsigned int, part.top));
    st_agent(mine + 1, (unsigned int)part.at);
    st_agent(mine + 2, __builtin_bit_cast(unsigned int, part.sum));
    // the last of the row's workgroups finds the others' parts stored; the
    // counter wraps to 0 for the next call
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
    const unsigned int before = __hip_atomic_fetch_add(counters + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before != (unsigned int)tiles - 1u) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    st_agent(counters + row, 0u);
    for (int t = 0; t < tiles; ++t) {
      const unsigned int *p = (const unsigned int *)(parts + (size_t)row * tiles + t);
      const LogitsPart q = {__builtin_bit_cast(float, ld_agent(p)), (int32_t)ld_agent(p + 1),
                            __builtin_bit_cast(float, ld_agent(p + 2)), 0.0f};
      part = t == 0 ? q : join(part, q);
    }
  }
  if (a.token) a.token[row] = part.at;
  if (a.lse) {
    float l = part.top;                          // -infinity, infinity or NaN as it is
    if (__builtin_fabsf(l) < __builtin_inff()) l += logf(part.sum);
    a.lse[row] = l;
  }
}

template <typename T> int launch_logits(const cortex_logits_t &a, int32_t *status, void *ws, void *stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool wide = a.logits_ld % V == 0 && aligned16(a.logits) && (!a.out || (a.out_ld % V == 0 && aligned16(a.out)));
  const dim3 grid((a.vocab + kLogitsTile - 1) / kLogitsTile, a.rows);
  uint32_t *counters = (uint32_t *)ws;
  LogitsPart *parts = (LogitsPart *)((char *)ws + kLogitsCounterBytes);
  if (wide) logits_kernel<T, V><<<grid, kLogitsThreads, 0, (hipStream_t)stream>>>(a, status, counters, parts);
  else logits_kernel<T, 1><<<grid, kLogitsThreads, 0, (hipStream_t)stream>>>(a, status, counters, parts);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

}  // namespace cortex

using namespace cortex;

extern "C" size_t cortex_logits_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || rows > kLogitsMaxRows || vocab < 1) return 0;
  return kLogitsCounterBytes + (size_t)rows * (((size_t)vocab + kLogitsTile - 1) / kLogitsTile) * sizeof(LogitsPart);
}

extern "C" int cortex_logits_process(const cortex_logits_t *args, int32_t *d_status, void *d_ws, size_t ws_bytes,
                                     void *stream) {
  if (!args || !d_status || !d_ws) return CORTEX_E_INVAL;
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
