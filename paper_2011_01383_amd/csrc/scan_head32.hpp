// Prompts of the scan with one decay per head, float32: the products of
// scan_head.hpp on the fp32 matrix units, over sub-chunks of 32 tokens.
//
// A 16x16x4 product takes one value per lane: index lane & 15, k = lane >> 4.
// Four of them, over sixteen k, are issued with k = 4 (lane >> 4) + i at step i
// for both operands, so four neighbouring values of a row, or of a result
// (rows 4 (lane >> 4) + 0..3), are the operands of the four steps as they
// stand: the state goes from accumulators into the output's products without
// moving.  At 64 lanes x 2 operations a cycle and SIMD these units bound it;
// three bf16 planes a value would take six products of a sixteenth of the time
// each, and the splitting of every value that is read.
#pragma once

#include "scan_head.hpp"

namespace cortex {

constexpr int kSub32 = 32;

template <int N> struct HeadLds32 {
  float B[kSub32][N + 4];        // rows 16 bytes longer: see the bf16 form
  float C[kSub32][N + 4];
  float x[kSub32][64 + 4];
  float M[kSub32][kSub32 + 4];   // scores [t][s]
  float dt[kSub32], cum[kSub32], grow[kSub32], weight[kSub32];
  float decay;
};

__device__ __forceinline__ float4 load4f(const float *p, bool wide) {
  return wide ? *(const float4 *)p : make_float4(p[0], p[1], p[2], p[3]);
}

template <int N, int PART>
__global__ void __launch_bounds__(kHeadThreads, 2) head_mfma32_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w,
                                                                      int Q, int wide) {
  constexpr int NT = N / 16, kItems = (N / 4 * kSub32 + kHeadThreads - 1) / kHeadThreads;
  __shared__ HeadLds32<N> lds;
  if (load_status(status) != 0) return;
  const int slot = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int q = lane >> 4, l16 = lane & 15;
  const int P = a.head_dim, blocks = (P + 63) / 64;
  const int head = (int)blockIdx.y / blocks, p0 = (int)blockIdx.y % blocks * 64;
  const int heads = a.channels / P, g = head / (heads / a.groups);
  int seq, begin, end;
  if constexpr (PART == 0) {
    seq = slot;
    if (blockIdx.y == 0) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, seq, status);
    begin = a.seq_offsets[seq];
    end = a.seq_offsets[seq + 1];
    if (begin < 0 || end < begin || end > a.num_tokens) return;
  } else {
    if (PART == 1 && blockIdx.y == 0) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, slot, status);
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
  const int pw = p0 + wave * 16;
  const bool works = pw < P;
  const int d = head * P + (works ? pw : 0) + l16;

  f32x4 h[NT];
  const float *h_in = PART == 2 ? w.state + ((int64_t)slot * a.channels + d) * N
                                : PART == 0 && row >= 0 && a.state_in ? a.state_in + ((int64_t)row * a.channels + d) * N : nullptr;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    h[nt] = works && h_in ? *(const f32x4 *)(h_in + nt * 16 + q * 4) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float A2 = a.A[head] * kLog2e, bias = a.dt_bias ? a.dt_bias[head] : 0.0f, skip = a.skip ? a.skip[head] : 0.0f;
  const float *xs = (const float *)a.x + head * P + p0, *ds = (const float *)a.dt + head;
  const float *Bs = (const float *)a.B + g * N, *Cs = (const float *)a.C + g * N;
  const float *zs = a.z ? (const float *)a.z + d : nullptr;
  float *ys = (float *)a.y + d;
  float steps = 0.0f;

  const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float4 xr[2], br[kItems], cr[kItems];
  float raw = 0.0f;
  auto fetch = [&](int t0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = i * kHeadThreads + tid, c = id % 16 * 4;
      const int64_t t = t0 + id / 16;
      xr[i] = t < end && p0 + c < P ? load4f(xs + t * a.x_ld + c, wide & 1) : none;
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid, c = id % (N / 4) * 4;
      const int64_t t = t0 + id / (N / 4);
      const bool in = t < end && id < N / 4 * kSub32;
      br[i] = in ? load4f(Bs + t * a.B_ld + c, wide & 2) : none;
      if (PART != 1) cr[i] = in ? load4f(Cs + t * a.C_ld + c, wide & 4) : none;
    }
    raw = lane < kSub32 && t0 + lane < end ? ds[(int64_t)(t0 + lane) * a.dt_ld] : 0.0f;
  };

  if (begin < end) fetch(begin);
#pragma unroll 1
  for (int t0 = begin; t0 < end; t0 += kSub32) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int id = i * kHeadThreads + tid;
      *(float4 *)&lds.x[id / 16][id % 16 * 4] = xr[i];
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid;
      if (id < N / 4 * kSub32) {
        *(float4 *)&lds.B[id / (N / 4)][id % (N / 4) * 4] = br[i];
        if (PART != 1) *(float4 *)&lds.C[id / (N / 4)][id % (N / 4) * 4] = cr[i];
      }
    }
    if (wave == 0) {
      const float dt = lane < kSub32 && t0 + lane < end ? step_size(a, raw, bias) : 0.0f;
      const float la = dt * A2;
      float up = la, down = la;                  // from the start, and from the end: see the bf16 form
#pragma unroll
      for (int m = 1; m < kSub32; m <<= 1) {
        const float u = __shfl_up(up, m), v = __shfl_down(down, m);
        if (lane >= m) up += u;
        if (lane + m < kSub32) down += v;
      }
      const float after = __shfl_down(down, 1);
      if (lane < kSub32) {
        lds.dt[lane] = dt;
        lds.cum[lane] = up;
        lds.grow[lane] = fast_exp2(up);
        lds.weight[lane] = fast_exp2(lane == kSub32 - 1 ? 0.0f : after) * dt;
      }
      if (lane == 0) lds.decay = fast_exp2(down);
      if (PART == 1) {
        float sum = dt;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        steps += sum;
      }
    }
    __syncthreads();
    if (t0 + kSub32 < end) fetch(t0 + kSub32);

    // the wave's channels of x, by sixteen tokens: k = 4 q + i
    float x[2][4];
#pragma unroll
    for (int si = 0; si < 2; ++si)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[si][i] = lds.x[si * 16 + q * 4 + i][wave * 16 + l16];

    if constexpr (PART != 1) {
      float zr[2][4];
      if (zs && works)
#pragma unroll
        for (int ti = 0; ti < 2; ++ti)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + ti * 16 + q * 4 + i;
            zr[ti][i] = t < end ? zs[t * a.z_ld] : 0.0f;
          }
      if (wave < 3) {                            // tiles (0,0) (1,0) (1,1) of the scores
        const int ti = wave > 0, si = wave > 1;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int m = 0; m < NT; ++m)
          acc = mfma_k16(*(const float4 *)&lds.B[si * 16 + l16][m * 16 + q * 4], *(const float4 *)&lds.C[ti * 16 + l16][m * 16 + q * 4], acc);
        const int t = ti * 16 + l16, s = si * 16 + q * 4;
        const float ct = lds.cum[t];
        const f32x4 cs = *(const f32x4 *)&lds.cum[s], dt = *(const f32x4 *)&lds.dt[s];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = s + i <= t ? acc[i] * (fast_exp2(ct - cs[i]) * dt[i]) : 0.0f;
        *(f32x4 *)&lds.M[t][s] = acc;
      }
      f32x4 y[2];
#pragma unroll
      for (int ti = 0; ti < 2; ++ti) y[ti] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (works) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float4 hv = make_float4(h[nt][0], h[nt][1], h[nt][2], h[nt][3]);
#pragma unroll
          for (int ti = 0; ti < 2; ++ti) y[ti] = mfma_k16(*(const float4 *)&lds.C[ti * 16 + l16][nt * 16 + q * 4], hv, y[ti]);
        }
#pragma unroll
        for (int ti = 0; ti < 2; ++ti) y[ti] *= *(const f32x4 *)&lds.grow[ti * 16 + q * 4];
      }
      __syncthreads();                           // the scores are there
      if (works) {
        // an infinite or NaN x: as in the bf16 form
        float xf[2][4];
        int first_odd = kSub32;
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
          for (int ti = si; ti < 2; ++ti)
            y[ti] = mfma_k16(*(const float4 *)&lds.M[ti * 16 + l16][si * 16 + q * 4],
                             make_float4(xf[si][0], xf[si][1], xf[si][2], xf[si][3]), y[ti]);
#pragma unroll
        for (int ti = 0; ti < 2; ++ti)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + ti * 16 + q * 4 + i;
            float v = __builtin_fmaf(skip, x[ti][i], y[ti][i]);
            if (ti * 16 + q * 4 + i >= first_odd) v = __builtin_nanf("");
            if (zs) v *= silu(zr[ti][i]);
            if (t < end) ys[t * a.y_ld] = v;
          }
      }
    }
    if (works) {
      const float decay = lds.decay;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) h[nt] *= decay;
#pragma unroll
      for (int si = 0; si < 2; ++si) {
        const f32x4 ws = *(const f32x4 *)&lds.weight[si * 16 + q * 4];
        const float4 xw = make_float4(x[si][0] * ws[0], x[si][1] * ws[1], x[si][2] * ws[2], x[si][3] * ws[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float *b = &lds.B[si * 16 + q * 4][nt * 16 + l16];
          h[nt] = mfma_k16(make_float4(b[0], b[N + 4], b[2 * (N + 4)], b[3 * (N + 4)]), xw, h[nt]);
        }
      }
    }
  }
  if (PART == 1 && tid == 0 && p0 == 0) w.steps[(int64_t)slot * heads + head] = steps;
  float *h_out = PART == 1 ? w.state + ((int64_t)slot * a.channels + d) * N
                           : PART == 0 && row >= 0 && a.state_out ? a.state_out + ((int64_t)row * a.channels + d) * N : nullptr;
  if (works && h_out)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) *(f32x4 *)(h_out + nt * 16 + q * 4) = h[nt];
}

}  // namespace cortex
