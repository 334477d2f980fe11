// Causal depthwise convolution over time, for prompts and for single tokens.
//
// A thread owns V neighbouring channels (16 bytes of them, or one where rows do
// not start at 16-byte boundaries) and Q consecutive tokens.  It loads their
// inputs and the W - 1 before them at once, then slides the window down them.
// The bytes of x and y bound it: 2 W + 4 operations per element loaded and stored.
// 8,192 tokens of 2,304 bf16 channels: 24 us, 3.2 TB/s of inputs and outputs (a
// large copy runs at 4.8); 7 rows of single tokens: 3.7 us.  What is left is the
// shape of the launch: a wave looks up its sequence and pool row, loads its rows
// and weights, then stores, once, and all waves do so at the same time (chunks of
// 8 to 16 tokens measure the same).
#include "sequence.hpp"

namespace cortex {

constexpr int kConvThreads = 64;

template <typename T, int W, int V, int Q, bool STEP>
__global__ void __launch_bounds__(kConvThreads) conv_kernel(cortex_conv_t a, int32_t *status) {
  if (entry_status(status) != 0) return;
  const int slot = (int)blockIdx.x;
  Chunk c;
  if constexpr (STEP) {
    c.seq = c.first = c.begin = slot;
    c.last = c.end = slot + 1;
  } else {
    if (blockIdx.y == 0) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, slot, status);
    c = find_chunk(a.seq_offsets, a.num_seqs, a.num_tokens, Q, slot);
    if (c.seq < 0) return;
  }
  const int ch = ((int)blockIdx.y * kConvThreads + (int)threadIdx.x) * V;
  const bool starts = c.begin == c.first;
  int row = -1;
  if (starts && (a.state_in || a.state_out)) {
    row = state_row(a.state_index, c.seq, a.state_rows, status);
    if (row < -1) return;
  }
  if (ch >= a.channels) return;

  const T *x = (const T *)a.x + ch;
  T *y = (T *)a.y + ch;
  const int64_t state_at = (int64_t)row * (W - 1) * a.channels + ch;
  // in[k]: the input of row begin - (W - 1) + k
  typedef T vec __attribute__((ext_vector_type(V)));
  vec in[Q + W - 1];
#pragma unroll
  for (int k = 0; k < Q + W - 1; ++k) {
    const int t = c.begin - (W - 1) + k, at = t < c.first ? c.first : t < c.end ? t : c.end - 1;
    in[k] = (vec)(T)0.0f;
    if (c.begin < c.end) in[k] = *(const vec *)(x + (int64_t)at * a.x_ld);
  }
  float w[W][V], bias[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    bias[i] = a.bias ? a.bias[ch + i] : 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) w[k][i] = a.weight[(int64_t)(ch + i) * W + k];
  }
  // before the sequence's first token: its state, or zeros
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    if (c.begin - (W - 1) + k < c.first) {
      in[k] = (vec)(T)0.0f;
      // (a chunk is no shorter than the window: only a sequence's first reaches back here)
      if (a.state_in && row >= 0)
        in[k] = *(const vec *)((const T *)a.state_in + state_at + (int64_t)k * a.channels);
    }
  }
  if (starts && row >= 0 && a.state_out) {
    // The sequence's last W - 1 inputs.  The old state is loaded already, so the
    // pool may be updated in place.
    const int len = c.last - c.first;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
      const int j = len - (W - 1) + k;
      vec v = in[0];
      if (j >= 0) {
        v = *(const vec *)(x + (int64_t)(c.first + j) * a.x_ld);
      } else {
#pragma unroll
        for (int m = 1; m < W - 1; ++m)
          if (m == W - 1 + j) v = in[m];
      }
      *(vec *)((T *)a.state_out + state_at + (int64_t)k * a.channels) = v;
    }
  }
#pragma unroll
  for (int j = 0; j < Q; ++j) {
    const int t = c.begin + j;
    if (t < c.end) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[i] = bias[i];
#pragma unroll
        for (int k = 0; k < W; ++k) v[i] = __builtin_fmaf(w[k][i], to_float<T>(in[j + k][i]), v[i]);
        if (a.silu) v[i] = silu(v[i]);
      }
      Pack<T, V>::store(y + (int64_t)t * a.y_ld, v);
    }
  }
}

template <typename T, int W, int V, int Q, bool STEP>
int launch_conv(const cortex_conv_t &a, int32_t *status, void *stream) {
  static_assert(STEP || Q >= W - 1, "a sequence's second chunk must not reach its state");
  const int64_t slots = STEP ? a.num_seqs : chunk_slots(a.num_tokens, a.num_seqs, Q);
  const int tiles = (a.channels / V + kConvThreads - 1) / kConvThreads;
  conv_kernel<T, W, V, Q, STEP><<<dim3((unsigned)slots, tiles), kConvThreads, 0, (hipStream_t)stream>>>(a, status);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

// Sixteen tokens a thread, so that the W - 1 inputs before them are a fifth more to
// read; four while sixteen would leave SIMDs (1,024) with less than two waves.
template <typename T, int W, int V> int launch_conv_chunks(const cortex_conv_t &a, int32_t *status, void *stream) {
  const int64_t waves = chunk_slots(a.num_tokens, a.num_seqs, 16) * ((a.channels / V + kConvThreads - 1) / kConvThreads);
  return waves >= 2048 ? launch_conv<T, W, V, 16, false>(a, status, stream) : launch_conv<T, W, V, 4, false>(a, status, stream);
}

template <typename T, int W, bool STEP> int launch_conv_width(const cortex_conv_t &a, int32_t *status, void *stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool wide = a.channels % V == 0 && a.x_ld % V == 0 && a.y_ld % V == 0 && aligned16(a.x) && aligned16(a.y) &&
                    aligned16(a.state_in) && aligned16(a.state_out);
  if constexpr (STEP)
    return wide ? launch_conv<T, W, V, 1, true>(a, status, stream) : launch_conv<T, W, 1, 1, true>(a, status, stream);
  else
    return wide ? launch_conv_chunks<T, W, V>(a, status, stream) : launch_conv_chunks<T, W, 1>(a, status, stream);
}

template <typename T, bool STEP> int launch_conv_typed(const cortex_conv_t &a, int32_t *status, void *stream) {
  if (a.width == 2) return launch_conv_width<T, 2, STEP>(a, status, stream);
  if (a.width == 3) return launch_conv_width<T, 3, STEP>(a, status, stream);
  return launch_conv_width<T, 4, STEP>(a, status, stream);
}

static int conv_entry(const cortex_conv_t *a, bool step, int32_t *status, void *stream) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (bad_batch(a->dtype, a->num_seqs, a->num_tokens, a->channels, a->state_rows, a->state_index,
                a->state_in || a->state_out))
    return CORTEX_E_INVAL;
  if (a->width < 2 || a->width > 4) return CORTEX_E_INVAL;
  if (step ? a->num_tokens != a->num_seqs : !a->seq_offsets) return CORTEX_E_INVAL;
  if (!a->weight || a->x_ld < a->channels || a->y_ld < a->channels) return CORTEX_E_INVAL;
  if (a->num_tokens > 0 && (!a->x || !a->y)) return CORTEX_E_INVAL;
  if (a->num_seqs == 0) return a->num_tokens == 0 ? CORTEX_OK : CORTEX_E_INVAL;
  if (a->dtype == CORTEX_BF16)
    return step ? launch_conv_typed<bf16_t, true>(*a, status, stream) : launch_conv_typed<bf16_t, false>(*a, status, stream);
  return step ? launch_conv_typed<float, true>(*a, status, stream) : launch_conv_typed<float, false>(*a, status, stream);
}

}  // namespace cortex

extern "C" int cortex_conv_forward(const cortex_conv_t *args, int32_t *d_status, void *stream) {
  return cortex::conv_entry(args, false, d_status, stream);
}
extern "C" int cortex_conv_step(const cortex_conv_t *args, int32_t *d_status, void *stream) {
  return cortex::conv_entry(args, true, d_status, stream);
}
