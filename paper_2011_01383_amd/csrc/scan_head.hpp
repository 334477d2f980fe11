// Prompts of the scan with one decay per head, as matrix products (bf16).
//
// Within a sub-chunk of 64 tokens, with c_t = sum_{s <= t} dt_s A and the state
// h that enters it,
//   y_t  = sum_{s <= t} (C_t . B_s) exp(c_t - c_s) dt_s x_s  +  exp(c_t) C_t h
//   h'   = exp(c_63) h + sum_s exp(c_63 - c_s) dt_s x_s B_s
// A workgroup takes 64 channels of one head (a wave 16 of them) and walks the
// sub-chunks of a segment with the state in its accumulators, so no state goes
// to memory between them.
//
// Precision.  x, B and C are bf16 and enter the matrix units as they are.  What
// is computed on the way is split into bf16 planes (each the rounding of what
// the ones before it leave): the scaled scores and the state that y reads into
// two, 16 bits, since y itself is rounded to bf16; the step-weighted x that the
// state is summed from into three, all 24 bits, since the state stays float32.
// All sums are float32.  An infinite or NaN x makes its channel NaN from its token
// on (the token-by-token order might keep an infinity).
//
// Layouts.  A 16x16x32 product takes both operands as (index = lane & 15; 8
// consecutive k from 8 (lane >> 4)) and leaves its result as (column = lane &
// 15; rows 4 (lane >> 4) + 0..3).  The order of k is free as long as both
// operands agree, so every array over tokens or state entries that is summed
// over keeps position 8 q + 4 a + r for element 16 a + 4 q + r of each 32: a
// result then is an operand of the next product as it stands.  The scores are
// computed as B C^T (columns t) and the state as [N, channels], so neither is
// ever transposed; B and x are, on their way into LDS.
#pragma once

#include "sequence.hpp"

namespace cortex {

typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4v __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kSub = 64;                 // tokens of a sub-chunk
constexpr int kHeadWaves = 4;
constexpr int kHeadThreads = 64 * kHeadWaves;

__device__ __forceinline__ f32x4 mfma_bf16x32(bf16x8v a, bf16x8v b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Position of element e in the order described above.
__device__ __forceinline__ constexpr int k_position(int e) {
  return (e & ~31) | ((e & 12) << 1) | ((e & 16) >> 2) | (e & 3);
}

// The next bf16 plane of v, which keeps what is left.
template <int M> __device__ __forceinline__ void plane(float (&v)[M], __bf16 (&p)[M]) {
#pragma unroll
  for (int i = 0; i < M; ++i) {
    p[i] = (__bf16)v[i];
    v[i] -= (float)p[i];
  }
}
__device__ __forceinline__ bf16x8v pack8(const __bf16 (&p)[8]) {
  return bf16x8v{p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]};
}

// LDS of one workgroup.  The scores take the place of B's rows once those are read.
template <int N> struct HeadLds {
  static constexpr int NP = N < 32 ? 32 : N;      // the products over N take 32 at a time; what is past N is 0
  static constexpr int kRow = NP + 8;             // rows 16 bytes longer: 8 lanes' 16-byte reads cover all banks
  static constexpr int kTok = kSub + 8;
  union {
    unsigned short B[kSub][kRow];                 // [s][n position]
    unsigned short M[2][kSub][kTok];              // scores, two planes: [t][s position]
  };
  unsigned short C[kSub][kRow];                   // [t][n position]
  unsigned short BT[N][kTok];                     // [n][s position]
  unsigned short xT[64][kTok];                    // [channel][s position]
  float dt[kSub], cum[kSub], grow[kSub], weight[kSub];   // dt_s, c_t, exp(c_t), exp(c_63 - c_s) dt_s
  float decay;                                    // exp(c_63)
};

__device__ __forceinline__ bf16x8v lds8(const unsigned short *p) { return __builtin_bit_cast(bf16x8v, *(const u32x4v *)p); }

// Eight elements of a row, as one load where the address allows it.
__device__ __forceinline__ u32x4v load8(const bf16_t *p, bool wide) {
  if (wide) return *(const u32x4v *)p;
  const unsigned short *s = (const unsigned short *)p;
  u32x4v r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (unsigned int)s[2 * i] | (unsigned int)s[2 * i + 1] << 16;
  return r;
}

// Two rows of eight elements, of neighbouring tokens: their pairs, one word per element.
__device__ __forceinline__ unsigned int pair_of(const u32x4v &a, const u32x4v &b, int i) {
  const unsigned int x = a[i / 2], y = b[i / 2];
  return i & 1 ? (x >> 16) | (y & 0xffff0000u) : (x & 0xffffu) | y << 16;
}

// PART as for the channel scan: 0 whole sequences, 1 a segment's state from
// zero, 2 outputs from the state that enters it.
template <int N, int PART>
__global__ void __launch_bounds__(kHeadThreads, 2) head_mfma_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w,
                                                                    int Q, int wide) {
  typedef HeadLds<N> Lds;
  constexpr int NT = N / 16, NB = Lds::NP / 32;
  constexpr int OL = N / 8 < 4 ? N / 8 : 4;                       // octets of a row that neighbouring lanes take
  constexpr int kItems = (N / 8 * 32 + kHeadThreads - 1) / kHeadThreads;   // (octet, pair of tokens) per thread
  __shared__ Lds lds;
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
  const int pw = p0 + wave * 16;                 // the wave's channels in the head
  const bool works = pw < P;                     // a head of less than 64 channels has none for the last waves
  const int d = head * P + (works ? pw : 0) + l16;

  f32x4 h[NT];                                   // rows n = 16 nt + 4 q + 0..3, column channel l16
  const float *h_in = PART == 2 ? w.state + ((int64_t)slot * a.channels + d) * N
                                : PART == 0 && row >= 0 && a.state_in ? a.state_in + ((int64_t)row * a.channels + d) * N : nullptr;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    h[nt] = works && h_in ? *(const f32x4 *)(h_in + nt * 16 + q * 4) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float A2 = a.A[head] * kLog2e, bias = a.dt_bias ? a.dt_bias[head] : 0.0f, skip = a.skip ? a.skip[head] : 0.0f;
  const bf16_t *xs = (const bf16_t *)a.x + head * P + p0, *ds = (const bf16_t *)a.dt + head;
  const bf16_t *Bs = (const bf16_t *)a.B + g * N, *Cs = (const bf16_t *)a.C + g * N;
  const bf16_t *zs = a.z ? (const bf16_t *)a.z + d : nullptr;
  bf16_t *ys = (bf16_t *)a.y + d;
  float steps = 0.0f;

  // What the next sub-chunk needs, loaded while this one is worked on.  Tokens
  // past the segment's end are zeros, with no step.
  u32x4v xr[2], br[kItems][2], cr[kItems][2];
  float raw = 0.0f;
  const u32x4v none = {0, 0, 0, 0};
  auto fetch = [&](int t0) {
    const int xo = tid & 3 | tid >> 7 << 2, xp = tid >> 2 & 31;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int64_t t = t0 + 2 * xp + r;
      xr[r] = t < end && p0 + xo * 8 < P ? load8(xs + t * a.x_ld + xo * 8, wide & 1) : none;
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid, o = id % OL + id / (OL * 32) * OL, sp = id / OL % 32;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int64_t t = t0 + 2 * sp + r;
        const bool in = t < end && o < N / 8;
        br[i][r] = in ? load8(Bs + t * a.B_ld + o * 8, wide & 2) : none;
        if (PART != 1) cr[i][r] = in ? load8(Cs + t * a.C_ld + o * 8, wide & 4) : none;
      }
    }
    raw = t0 + lane < end ? to_float<bf16_t>(ds[(int64_t)(t0 + lane) * a.dt_ld]) : 0.0f;
  };
  // Rows of eight state entries (octet o) in k order: two halves of 8 bytes.
  auto put_row = [&](unsigned short *to, int o, const u32x4v &v) {
    const int e = o * 8;
    *(uint2 *)(to + k_position(e)) = make_uint2(v[0], v[1]);
    *(uint2 *)(to + k_position(e + 4)) = make_uint2(v[2], v[3]);
  };
  if constexpr (N < 32)
    for (int i = tid; i < kSub * (Lds::NP - N) / 4; i += kHeadThreads) {
      const int s = i / ((Lds::NP - N) / 4), e = N + i % ((Lds::NP - N) / 4) * 4;
      *(uint2 *)&lds.C[s][k_position(e)] = make_uint2(0, 0);
    }

  if (begin < end) fetch(begin);
#pragma unroll 1
  for (int t0 = begin; t0 < end; t0 += kSub) {
    __syncthreads();                             // everyone is done with the last sub-chunk's LDS
    {
      const int xo = tid & 3 | tid >> 7 << 2, xp = k_position(2 * (tid >> 2 & 31));
#pragma unroll
      for (int i = 0; i < 8; ++i) *(unsigned int *)&lds.xT[xo * 8 + i][xp] = pair_of(xr[0], xr[1], i);
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid, o = id % OL + id / (OL * 32) * OL, s = id / OL % 32 * 2;
      if (o < N / 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k) *(unsigned int *)&lds.BT[o * 8 + k][k_position(s)] = pair_of(br[i][0], br[i][1], k);
        if (PART != 1) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            put_row(lds.B[s + r], o, br[i][r]);
            put_row(lds.C[s + r], o, cr[i][r]);
          }
        }
      }
    }
    if constexpr (PART != 1 && N < 32)                     // the scores were here
      for (int i = tid; i < kSub * (Lds::NP - N) / 4; i += kHeadThreads) {
        const int s = i / ((Lds::NP - N) / 4), e = N + i % ((Lds::NP - N) / 4) * 4;
        *(uint2 *)&lds.B[s][k_position(e)] = make_uint2(0, 0);
      }
    if (wave == 0) {
      // a lane is a token.  The weights of the state come from a sum from the
      // end: those near the end, which count most, are sums of few terms
      const float dt = t0 + lane < end ? step_size(a, raw, bias) : 0.0f;
      const float la = dt * A2;
      float up = la, down = la;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const float u = __shfl_up(up, m), v = __shfl_down(down, m);
        if (lane >= m) up += u;
        if (lane + m < 64) down += v;
      }
      const float after = __shfl_down(down, 1);
      lds.dt[lane] = dt;
      lds.cum[lane] = up;
      lds.grow[lane] = fast_exp2(up);
      lds.weight[lane] = fast_exp2(lane == 63 ? 0.0f : after) * dt;
      if (lane == 0) lds.decay = fast_exp2(down);
      if (PART == 1) {
        float sum = dt;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        steps += sum;
      }
    }
    __syncthreads();
    if (t0 + kSub < end) fetch(t0 + kSub);

    if constexpr (PART != 1) {
      bf16_t zr[4][4];
      if (zs && works)
#pragma unroll
        for (int ti = 0; ti < 4; ++ti)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + ti * 16 + q * 4 + i;
            zr[ti][i] = t < end ? zs[t * a.z_ld] : (bf16_t)0.0f;
          }
      // Scores: 10 tiles of 16 x 16 on and below the diagonal, and the two above it that a
      // product over 32 tokens reaches: three a wave.
      u16x4 m0[3], m1[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int id = wave + 4 * k;
        // (0,0) (1,0) (1,1) (2,0) (2,1) (2,2) (3,0) (3,1) (3,2) (3,3), then (0,1) (2,3)
        const int ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : id < 10 ? 3 : id == 10 ? 0 : 2;
        const int si = id < 10 ? id - ti * (ti + 1) / 2 : id == 10 ? 1 : 3;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        if (id < 10) {
#pragma unroll
          for (int m = 0; m < NB; ++m)
            acc = mfma_bf16x32(lds8(&lds.B[si * 16 + l16][m * 32 + q * 8]), lds8(&lds.C[ti * 16 + l16][m * 32 + q * 8]), acc);
          const int t = ti * 16 + l16, s = si * 16 + q * 4;
          const float ct = lds.cum[t];
          const f32x4 cs = *(const f32x4 *)&lds.cum[s], dt = *(const f32x4 *)&lds.dt[s];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] = s + i <= t ? acc[i] * (fast_exp2(ct - cs[i]) * dt[i]) : 0.0f;
        }
        float v[4] = {acc[0], acc[1], acc[2], acc[3]};
        __bf16 b[4];
        plane(v, b);
        m0[k] = __builtin_bit_cast(u16x4, b);
        plane(v, b);
        m1[k] = __builtin_bit_cast(u16x4, b);
      }
      __syncthreads();                           // B's rows are read
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int id = wave + 4 * k;
        const int ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : id < 10 ? 3 : id == 10 ? 0 : 2;
        const int si = id < 10 ? id - ti * (ti + 1) / 2 : id == 10 ? 1 : 3;
        *(u16x4 *)&lds.M[0][ti * 16 + l16][k_position(si * 16 + q * 4)] = m0[k];
        *(u16x4 *)&lds.M[1][ti * 16 + l16][k_position(si * 16 + q * 4)] = m1[k];
      }
      // From the state: rows t, columns channels.
      f32x4 y[4];
#pragma unroll
      for (int ti = 0; ti < 4; ++ti) y[ti] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (works) {
#pragma unroll
        for (int m = 0; m < NB; ++m) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = h[2 * m][i];
            v[4 + i] = 2 * m + 1 < NT ? h[2 * m + 1 < NT ? 2 * m + 1 : 0][i] : 0.0f;
          }
          __bf16 b[8];
          plane(v, b);
          const bf16x8v hi = pack8(b);
          plane(v, b);
          const bf16x8v lo = pack8(b);
#pragma unroll
          for (int ti = 0; ti < 4; ++ti) {
            const bf16x8v c = lds8(&lds.C[ti * 16 + l16][m * 32 + q * 8]);
            y[ti] = mfma_bf16x32(c, lo, y[ti]);
            y[ti] = mfma_bf16x32(c, hi, y[ti]);
          }
        }
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
          const f32x4 e = *(const f32x4 *)&lds.grow[ti * 16 + q * 4];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[ti][i] *= e[i];
        }
      }
      __syncthreads();                           // the scores are there
      if (works) {
        bf16x8v x[2];
        unsigned int odd = 0;                    // an infinity or NaN: an exponent of all ones
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          x[kb] = lds8(&lds.xT[wave * 16 + l16][kb * 32 + q * 8]);
          const u32x4v v = __builtin_bit_cast(u32x4v, x[kb]);
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= ((v[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        }
        // The products with the zeros above the diagonal would carry such an input to the tokens
        // before it.  It is left out of them, and its channel's tokens from its own on become NaN.
        int first_odd = kSub;
        if (__any(odd != 0)) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float v = (float)x[kb][j];
              if (!(__builtin_fabsf(v) < __builtin_inff())) {
                const int s = kb * 32 + (j < 4 ? 0 : 12) + q * 4 + j;
                first_odd = s < first_odd ? s : first_odd;
                x[kb][j] = (__bf16)0.0f;
              }
            }
          first_odd = min(first_odd, __shfl_xor(first_odd, 16));
          first_odd = min(first_odd, __shfl_xor(first_odd, 32));
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int ti = 2 * kb; ti < 4; ++ti) {
            y[ti] = mfma_bf16x32(lds8(&lds.M[1][ti * 16 + l16][kb * 32 + q * 8]), x[kb], y[ti]);
            y[ti] = mfma_bf16x32(lds8(&lds.M[0][ti * 16 + l16][kb * 32 + q * 8]), x[kb], y[ti]);
          }
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
          const u16x4 xv = *(const u16x4 *)&lds.xT[wave * 16 + l16][k_position(ti * 16 + q * 4)];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + ti * 16 + q * 4 + i;
            const unsigned short xb = xv[i];
            float v = __builtin_fmaf(skip, to_float<bf16_t>(__builtin_bit_cast(bf16_t, xb)), y[ti][i]);
            if (ti * 16 + q * 4 + i >= first_odd) v = __builtin_nanf("");
            if (zs) v *= silu(to_float<bf16_t>(zr[ti][i]));
            if (t < end) ys[t * a.y_ld] = from_float<bf16_t>(v);
          }
        }
      }
    }
    if (works) {
      const float decay = lds.decay;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) h[nt] *= decay;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8v x = lds8(&lds.xT[wave * 16 + l16][kb * 32 + q * 8]);
        const f32x4 w0 = *(const f32x4 *)&lds.weight[kb * 32 + q * 4], w1 = *(const f32x4 *)&lds.weight[kb * 32 + 16 + q * 4];
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = (float)x[i] * w0[i];
          v[4 + i] = (float)x[4 + i] * w1[i];
        }
        __bf16 b[8];
        plane(v, b);
        const bf16x8v x0 = pack8(b);
        plane(v, b);
        const bf16x8v x1 = pack8(b);
        plane(v, b);
        const bf16x8v x2 = pack8(b);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const bf16x8v bt = lds8(&lds.BT[nt * 16 + l16][kb * 32 + q * 8]);
          h[nt] = mfma_bf16x32(bt, x2, h[nt]);
          h[nt] = mfma_bf16x32(bt, x1, h[nt]);
          h[nt] = mfma_bf16x32(bt, x0, h[nt]);
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
