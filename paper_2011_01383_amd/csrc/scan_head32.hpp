// Prompts of the scan with one decay per head, float32: the products of
// scan_head.hpp on the fp32 matrix units, over sub-chunks of 32 tokens.
//
// A 16x16x4 product takes one value per lane: index lane & 15, k = lane >> 4.
// Four of them, over sixteen k, are issued with k = 4 (lane >> 4) + i at step i
// for both operands, so four neighbouring values of a row, or of a result
// (rows 4 (lane >> 4) + 0..3), are the operands of the four steps as they
// stand: the state goes from accumulators into the output's products without
// moving.  (Three bf16 planes a value, six products at a sixteenth of the time
// each, would want every value that is read split.)  4,099 tokens of 16 heads of 64
// channels, N = 64, in segments of 96: 15 + 10 + 29 us.  What bounds it there is the
// latency of three sub-chunks one after another: these units are busy a third of
// the time.
#pragma once

#include "scan_head.hpp"

namespace cortex {

template <int N> struct HeadLds32 {
  float B[kSub][N + 4];        // rows 16 bytes longer: see the bf16 form
  float C[kSub][N + 4];
  float x[kSub][64 + 4];
  float M[kSub][kSub + 4];   // scores [t][s]
  HeadSteps steps[4];
  float sums[kHeadWaves];
};

template <bool WIDE> __device__ __forceinline__ f32x4 load4f(const float *p) {
  if constexpr (WIDE) return *(const f32x4 *)p;
  return f32x4{p[0], p[1], p[2], p[3]};
}

// Sixteen k: the operands of four products.
__device__ __forceinline__ f32x4 mfma_k16(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

template <int N, int PART, bool WIDE>
__global__ void __launch_bounds__(kHeadThreads, 3) head_mfma32_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w, int Q,
                                                                    int64_t units) {
  constexpr int NT = N / 16, kItems = (N / 4 * kSub + kHeadThreads - 1) / kHeadThreads;
  __shared__ HeadLds32<N> lds;
  const int failed = entry_status(status);
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int q = lane >> 4, l16 = lane & 15;
  const int P = a.head_dim, blocks = (P + 63) / 64, heads = a.channels / P;
  const int64_t unit = unit_of_block(units);
  if (unit >= units) return;
  const int slot = (int)(unit / (heads * blocks)), part = (int)(unit % (heads * blocks));
  const int head = part / blocks, p0 = part % blocks * 64, g = head / (heads / a.groups);
  int seq, begin, end;
  if constexpr (PART == 0) {
    seq = slot;
    if (part == 0) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, seq, status);
    begin = a.seq_offsets[seq];
    end = a.seq_offsets[seq + 1];
    if (begin < 0 || end < begin || end > a.num_tokens) return;
  } else {
    if (PART == 1 && part == 0) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, slot, status);
    const Chunk c = find_chunk(a.seq_offsets, a.num_seqs, a.num_tokens, Q, slot);
    if (c.seq < 0 || c.begin == c.end) return;
    seq = c.seq;
    begin = c.begin;
    end = c.end;
  }
  int row = -1;
  if (PART == 0 && (a.state_in || a.state_out)) {
    row = state_row(a.state_index, seq, a.state_rows, status);
    if (row < -1) return;
  }
  if (__syncthreads_or(failed != 0)) return;     // all waves or none, as in the bf16 form
  const int pw = p0 + wave * 16;
  const bool works = pw < P;
  const int d = head * P + (works ? pw : 0) + l16;

  f32x4 h[NT];
  const float *h_in = PART == 2 ? w.state + ((int64_t)slot * a.channels + d) * N
                                : PART == 0 && row >= 0 && a.state_in ? a.state_in + ((int64_t)row * a.channels + d) * N : nullptr;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    h[nt] = works && h_in ? *(const f32x4 *)(h_in + nt * 16 + q * 4) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float A2 = decay_rate(a.A[head]), bias = a.dt_bias ? a.dt_bias[head] : 0.0f, skip = a.skip ? a.skip[head] : 0.0f;
  const float *xs = (const float *)a.x + head * P + p0, *ds = (const float *)a.dt + head;
  const float *Bs = (const float *)a.B + g * N, *Cs = (const float *)a.C + g * N;
  const int ch = head * P + (works ? pw : 0) + q * 4;
  const float *zs = a.z ? (const float *)a.z + ch : nullptr;
  float *ys = (float *)a.y + ch;
  float steps = 0.0f;

  const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
  f32x4 xr[2], br[kItems], cr[kItems];
  auto fetch = [&](int t0) {                      // as in the bf16 form
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = i * kHeadThreads + tid, c = p0 + id % 16 * 4 < P ? id % 16 * 4 : 0;
      xr[i] = load4f<WIDE>(xs + (int64_t)min(t0 + id / 16, end - 1) * a.x_ld + c);
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid, c = id % (N / 4) * 4;
      const int64_t t = min(t0 + id / (N / 4), end - 1);
      br[i] = load4f<WIDE>(Bs + t * a.B_ld + c);
      if (PART != 1) cr[i] = load4f<WIDE>(Cs + t * a.C_ld + c);
    }
  };
  auto raw_step = [&](int t0) { return ds[(int64_t)min(t0 + lane, end - 1) * a.dt_ld]; };
  auto make_steps = [&](int t0, int pair, float raw) {
    steps += put_steps(lds.steps, pair, lane, t0 + lane < end ? step_size(a, raw, bias) : 0.0f, A2);
  };

  if (begin < end) {
    fetch(begin);
    if (wave == 3) make_steps(begin, 0, raw_step(begin));
  }
#pragma unroll 1
  for (int t0 = begin, k = 0; t0 < end; t0 += kSub, ++k) {
    const bool makes = k % 2 == 0 && k / 2 % 4 == wave && t0 + 2 * kSub < end;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = i * kHeadThreads + tid;
      *(f32x4 *)&lds.x[id / 16][id % 16 * 4] = t0 + id / 16 < end ? xr[i] : none;
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid;
      const bool in = t0 + id / (N / 4) < end;
      if (id < N / 4 * kSub) {
        *(f32x4 *)&lds.B[id / (N / 4)][id % (N / 4) * 4] = in ? br[i] : none;
        if (PART != 1) *(f32x4 *)&lds.C[id / (N / 4)][id % (N / 4) * 4] = in ? cr[i] : none;
      }
    }
    __syncthreads();
    if (t0 + kSub < end) fetch(t0 + kSub);
    const float raw = makes ? raw_step(t0 + 2 * kSub) : 0.0f;
    const HeadSteps &st = lds.steps[k % 4];

    // the wave's channels of x, by sixteen tokens: k = 4 q + i
    float x[2][4];
#pragma unroll
    for (int si = 0; si < 2; ++si)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[si][i] = lds.x[si * 16 + q * 4 + i][wave * 16 + l16];

    if constexpr (PART != 1) {
      f32x4 zr[2];
      if (zs && works)
#pragma unroll
        for (int ti = 0; ti < 2; ++ti) zr[ti] = load4f<WIDE>(zs + (int64_t)min(t0 + ti * 16 + l16, end - 1) * a.z_ld);
      if (wave < 3) {                            // tiles (0,0) (1,0) (1,1) of the scores
        const int ti = wave > 0, si = wave > 1;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int m = 0; m < NT; ++m)
          acc = mfma_k16(*(const f32x4 *)&lds.B[si * 16 + l16][m * 16 + q * 4], *(const f32x4 *)&lds.C[ti * 16 + l16][m * 16 + q * 4], acc);
        const int t = ti * 16 + l16, s = si * 16 + q * 4;
        const f32x4 scale = step_scales(st, t, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i] = s + i <= t ? acc[i] * scale[i] : 0.0f;
          if (s + i == t) acc[i] += skip;
        }
        *(f32x4 *)&lds.M[t][s] = acc;
      }
      f32x4 y[2];
#pragma unroll
      for (int ti = 0; ti < 2; ++ti) y[ti] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (works) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int ti = 0; ti < 2; ++ti) y[ti] = mfma_k16(h[nt], *(const f32x4 *)&lds.C[ti * 16 + l16][nt * 16 + q * 4], y[ti]);
        }
#pragma unroll
        for (int ti = 0; ti < 2; ++ti) y[ti] *= st.grow[ti * 16 + l16];
      }
      __syncthreads();                           // the scores are there
      if (works) {
        // an infinite or NaN x: as in the bf16 form
        float xf[2][4];
        int first_odd = kSub;
#pragma unroll
        for (int si = 0; si < 2; ++si)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool fine = __builtin_fabsf(x[si][i]) < __builtin_inff();
            const int s = si * 16 + q * 4 + i;
            xf[si][i] = fine ? x[si][i] : 0.0f;
            first_odd = fine || first_odd < s ? first_odd : s;
          }
        first_odd = min(first_odd, __shfl_xor(first_odd, 16));
        first_odd = min(first_odd, __shfl_xor(first_odd, 32));
#pragma unroll
        for (int si = 0; si < 2; ++si)
#pragma unroll
          for (int ti = 0; ti < 2; ++ti)
            if (ti >= si)
              y[ti] = mfma_k16(f32x4{xf[si][0], xf[si][1], xf[si][2], xf[si][3]},
                               *(const f32x4 *)&lds.M[ti * 16 + l16][si * 16 + q * 4], y[ti]);
        if (__any(first_odd < kSub)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int odd = __shfl(first_odd, q * 4 + i);
#pragma unroll
            for (int ti = 0; ti < 2; ++ti)
              if (ti * 16 + l16 >= odd) y[ti][i] = __builtin_nanf("");
          }
        }
#pragma unroll
        for (int ti = 0; ti < 2; ++ti) {
          const int t = t0 + ti * 16 + l16;
          f32x4 v = y[ti];
          if (zs)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] *= silu(zr[ti][i]);
          if (t < end) {
            float *p = ys + (int64_t)t * a.y_ld;
            if constexpr (WIDE) {
              *(f32x4 *)p = v;
            } else {
              p[0] = v[0]; p[1] = v[1]; p[2] = v[2]; p[3] = v[3];
            }
          }
        }
      }
    }
    if (works) {
      const float decay = st.decay;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) h[nt] *= decay;
#pragma unroll
      for (int si = 0; si < 2; ++si) {
        const f32x4 ws = *(const f32x4 *)&st.weight[si * 16 + q * 4];
        const f32x4 xw = f32x4{x[si][0], x[si][1], x[si][2], x[si][3]} * ws;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float *b = &lds.B[si * 16 + q * 4][nt * 16 + l16];
          h[nt] = mfma_k16(f32x4{b[0], b[N + 4], b[2 * (N + 4)], b[3 * (N + 4)]}, xw, h[nt]);
        }
      }
    }
    if (makes) make_steps(t0 + 2 * kSub, (k / 2 + 1) % 2, raw);
  }
  if (PART == 1) {
    if (lane == 0) lds.sums[wave] = steps;
    __syncthreads();
    if (tid == 0 && p0 == 0)
      w.steps[(int64_t)slot * heads + head] = (lds.sums[0] + lds.sums[1]) + (lds.sums[2] + lds.sums[3]);
  }
  float *h_out = PART == 1 ? w.state + ((int64_t)slot * a.channels + d) * N
                           : PART == 0 && row >= 0 && a.state_out ? a.state_out + ((int64_t)row * a.channels + d) * N : nullptr;
  if (works && h_out)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) *(f32x4 *)(h_out + nt * 16 + q * 4) = h[nt];
}

}  // namespace cortex
