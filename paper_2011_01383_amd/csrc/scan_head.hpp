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
// ever transposed; B and x are, on their way into LDS.  y has channels as rows,
// so a lane loads z and stores y four channels at a time.
//
// What it does per sub-chunk and wave at N = 128: 102 products (1,632 cycles of
// a SIMD's matrix unit), about 60 16-byte reads of LDS.  The skip connection is
// the scores' diagonal.  Step sizes and their sums are made a sub-chunk ahead by
// one wave, beside the others' products.
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

// Rows of W elements that are read 16 bytes a lane down neighbouring rows: the
// 16-byte pieces of a row are exchanged by its number, so that eight lanes' reads
// fall into different banks without padding (which would leave room for one
// workgroup a CU instead of two).
template <int W> __device__ __forceinline__ int swizzled(int row, int pos) {
  const int f = W >= 64 ? (row ^ row >> 3) & 7 : row >> 2 & 3;
  return row * W + (((pos >> 3) ^ f) << 3 | (pos & 7));
}

// Step sizes of a sub-chunk: dt_s, c_s, exp(c_s), exp(c_63 - c_s) dt_s, exp(c_63).
struct HeadSteps {
  float dt[kSub], cum[kSub], grow[kSub], weight[kSub], decay;
};

template <int N> struct HeadLds {
  static constexpr int NP = N < 32 ? 32 : N;      // the products over N take 32 at a time; what is past N is 0
  static constexpr int kTok = kSub + 8;           // rows 16 bytes longer, for the same purpose
  unsigned short B[kSub * NP];                    // [s][n position]
  unsigned short C[kSub * NP];                    // [t][n position]
  unsigned short M[2][kSub * kSub];               // scores, two planes: [t][s position]
  unsigned short BT[N][kTok];                     // [n][s position]
  unsigned short xT[64][kTok];                    // [channel][s position]
  HeadSteps steps[2];
};

// A lane is a token.  The state's weights come from a sum from the end: those
// near the end, which count most, are sums of few terms.  Returns the sum of dt.
__device__ __forceinline__ float put_steps(HeadSteps &to, int lane, float dt, float A2) {
  const float up = lane_sums(dt * A2);
  const float rev = __shfl(dt, 63 - lane);
  const float down = lane_sums(rev * A2);         // of tokens 63 - lane and on
  const float after = __shfl_up(down, 1);
  to.dt[lane] = dt;
  to.cum[lane] = up;
  to.grow[lane] = fast_exp2(up);
  to.weight[63 - lane] = fast_exp2(lane == 0 ? 0.0f : after) * rev;
  if (lane == 63) to.decay = fast_exp2(down);
  return wave_sum(dt);
}

__device__ __forceinline__ bf16x8v lds8(const unsigned short *p) { return __builtin_bit_cast(bf16x8v, *(const u32x4v *)p); }

// Eight elements of a row: one load where every row starts at a 16-byte boundary.
template <bool WIDE> __device__ __forceinline__ u32x4v load8(const bf16_t *p) {
  if constexpr (WIDE) return *(const u32x4v *)p;
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
template <int N, int PART, bool WIDE>
__global__ void __launch_bounds__(kHeadThreads, 2) head_mfma_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w, int Q) {
  typedef HeadLds<N> Lds;
  constexpr int NT = N / 16, NB = Lds::NP / 32;
  constexpr int OL = N / 8 < 4 ? N / 8 : 4;                       // octets of a row that neighbouring lanes take
  constexpr int kItems = (N / 8 * 32 + kHeadThreads - 1) / kHeadThreads;   // (octet, pair of tokens) per thread
  __shared__ Lds lds;
  if (entry_status(status) != 0) return;
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
  const int ch = head * P + (works ? pw : 0) + q * 4;             // the lane's four channels of y and z
  const bf16_t *zs = a.z ? (const bf16_t *)a.z + ch : nullptr;
  bf16_t *ys = (bf16_t *)a.y + ch;
  float steps = 0.0f;

  // What the next sub-chunk needs, loaded while this one is worked on.  The loads
  // are unconditional, so that nothing waits for one of them: tokens past the
  // segment's end repeat the last one, and are made zeros when they are stored.
  u32x4v xr[2], br[kItems][2], cr[kItems][2];
  float raw = 0.0f;
  const u32x4v none = {0, 0, 0, 0};
  const int xo = (tid & 3) | (tid >> 7) << 2, xp = 2 * (tid >> 2 & 31);
  auto item_octet = [&](int i) { return tid % OL + (i * kHeadThreads + tid) / (OL * 32) * OL; };
  auto item_token = [&](int i) { return 2 * ((i * kHeadThreads + tid) / OL % 32); };
  auto fetch = [&](int t0) {
    const bf16_t *px = xs + (p0 + xo * 8 < P ? xo * 8 : 0);
#pragma unroll
    for (int r = 0; r < 2; ++r) xr[r] = load8<WIDE>(px + (int64_t)min(t0 + xp + r, end - 1) * a.x_ld);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int o = min(item_octet(i), N / 8 - 1);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int64_t t = min(t0 + item_token(i) + r, end - 1);
        br[i][r] = load8<WIDE>(Bs + t * a.B_ld + o * 8);
        if (PART != 1) cr[i][r] = load8<WIDE>(Cs + t * a.C_ld + o * 8);
      }
    }
    if (wave == 3) raw = to_float<bf16_t>(ds[(int64_t)min(t0 + lane, end - 1) * a.dt_ld]);
  };
  // Rows of eight state entries (octet o) in k order: two halves of 8 bytes.
  auto put_row = [&](unsigned short *to, int row, int o, const u32x4v &v) {
    *(uint2 *)(to + swizzled<Lds::NP>(row, k_position(o * 8))) = make_uint2(v[0], v[1]);
    *(uint2 *)(to + swizzled<Lds::NP>(row, k_position(o * 8 + 4))) = make_uint2(v[2], v[3]);
  };
  if constexpr (N < 32)
    for (int i = tid; i < kSub * (Lds::NP - N) / 4; i += kHeadThreads) {
      const int s = i / ((Lds::NP - N) / 4), e = N + i % ((Lds::NP - N) / 4) * 4;
      *(uint2 *)&lds.B[swizzled<Lds::NP>(s, k_position(e))] = make_uint2(0, 0);
      *(uint2 *)&lds.C[swizzled<Lds::NP>(s, k_position(e))] = make_uint2(0, 0);
    }
  // the tiles above the diagonal that a product over 32 tokens reaches: (0,1) and (2,3)
  if (PART != 1) {
    const int t = (tid >> 7) * 32 + (tid & 15), s = (tid >> 7) * 32 + 16 + (tid >> 4 & 3) * 4;
    *(uint2 *)&lds.M[tid >> 6 & 1][swizzled<kSub>(t, k_position(s))] = make_uint2(0, 0);
  }

  if (begin < end) {
    fetch(begin);
    if (wave == 3) steps += put_steps(lds.steps[0], lane, begin + lane < end ? step_size(a, raw, bias) : 0.0f, A2);
  }
  int buf = 0;
#pragma unroll 1
  for (int t0 = begin; t0 < end; t0 += kSub, buf ^= 1) {
    __syncthreads();                             // everyone is done with the last sub-chunk's LDS
    if (t0 + kSub > end) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (t0 + xp + r >= end) xr[r] = none;
#pragma unroll
        for (int i = 0; i < kItems; ++i)
          if (t0 + item_token(i) + r >= end) {
            br[i][r] = none;
            if (PART != 1) cr[i][r] = none;
          }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) *(unsigned int *)&lds.xT[xo * 8 + i][k_position(xp)] = pair_of(xr[0], xr[1], i);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int o = item_octet(i), s = item_token(i);
      if (o < N / 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k) *(unsigned int *)&lds.BT[o * 8 + k][k_position(s)] = pair_of(br[i][0], br[i][1], k);
        if (PART != 1) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            put_row(lds.B, s + r, o, br[i][r]);
            put_row(lds.C, s + r, o, cr[i][r]);
          }
        }
      }
    }
    __syncthreads();
    if (t0 + kSub < end) fetch(t0 + kSub);
    const HeadSteps &st = lds.steps[buf];

    if constexpr (PART != 1) {
      uint2 zr[4];
      if (zs && works)
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
          const bf16_t *p = zs + (int64_t)min(t0 + ti * 16 + l16, end - 1) * a.z_ld;
          if constexpr (WIDE) {
            zr[ti] = *(const uint2 *)p;
          } else {
            const unsigned short *e = (const unsigned short *)p;
            zr[ti] = make_uint2(e[0] | (unsigned int)e[1] << 16, e[2] | (unsigned int)e[3] << 16);
          }
        }
      // Scores: 10 tiles of 16 x 16 on and below the diagonal, three or two a wave.
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int id = wave + 4 * k;             // (0,0) (1,0) (1,1) (2,0) (2,1) (2,2) (3,0) (3,1) (3,2) (3,3)
        const int ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3, si = id - ti * (ti + 1) / 2;
        if (id < 10) {
          f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int m = 0; m < NB; ++m)
            acc = mfma_bf16x32(lds8(&lds.B[swizzled<Lds::NP>(si * 16 + l16, m * 32 + q * 8)]),
                               lds8(&lds.C[swizzled<Lds::NP>(ti * 16 + l16, m * 32 + q * 8)]), acc);
          const int t = ti * 16 + l16, s = si * 16 + q * 4;
          const float ct = st.cum[t];
          const f32x4 cs = *(const f32x4 *)&st.cum[s], dt = *(const f32x4 *)&st.dt[s];
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = s + i <= t ? acc[i] * (fast_exp2(ct - cs[i]) * dt[i]) : 0.0f;
            if (s + i == t) v[i] += skip;
          }
          __bf16 b[4];
          plane(v, b);
          *(u16x4 *)&lds.M[0][swizzled<kSub>(t, k_position(s))] = __builtin_bit_cast(u16x4, b);
          plane(v, b);
          *(u16x4 *)&lds.M[1][swizzled<kSub>(t, k_position(s))] = __builtin_bit_cast(u16x4, b);
        }
      }
      // From the state: rows channels, columns t.
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
            const bf16x8v c = lds8(&lds.C[swizzled<Lds::NP>(ti * 16 + l16, m * 32 + q * 8)]);
            y[ti] = mfma_bf16x32(lo, c, y[ti]);
            y[ti] = mfma_bf16x32(hi, c, y[ti]);
          }
        }
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) y[ti] *= st.grow[ti * 16 + l16];
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
        const bool any_odd = __any(odd != 0);
        int first_odd[4] = {kSub, kSub, kSub, kSub};
        if (any_odd) {
          int first = kSub;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float v = (float)x[kb][j];
              if (!(__builtin_fabsf(v) < __builtin_inff())) {
                const int s = kb * 32 + (j < 4 ? 0 : 12) + q * 4 + j;
                first = s < first ? s : first;
                x[kb][j] = (__bf16)0.0f;
              }
            }
          first = min(first, __shfl_xor(first, 16));
          first = min(first, __shfl_xor(first, 32));
#pragma unroll
          for (int i = 0; i < 4; ++i) first_odd[i] = __shfl(first, q * 4 + i);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int ti = 0; ti < 4; ++ti)
            if (ti >= 2 * kb) {
              y[ti] = mfma_bf16x32(x[kb], lds8(&lds.M[1][swizzled<kSub>(ti * 16 + l16, kb * 32 + q * 8)]), y[ti]);
              y[ti] = mfma_bf16x32(x[kb], lds8(&lds.M[0][swizzled<kSub>(ti * 16 + l16, kb * 32 + q * 8)]), y[ti]);
            }
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
          const int t = t0 + ti * 16 + l16;
          float v[4] = {y[ti][0], y[ti][1], y[ti][2], y[ti][3]};
          if (any_odd)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ti * 16 + l16 >= first_odd[i] ? __builtin_nanf("") : v[i];
          if (zs) {
            v[0] *= silu(__builtin_bit_cast(float, zr[ti].x << 16));
            v[1] *= silu(__builtin_bit_cast(float, zr[ti].x & 0xffff0000u));
            v[2] *= silu(__builtin_bit_cast(float, zr[ti].y << 16));
            v[3] *= silu(__builtin_bit_cast(float, zr[ti].y & 0xffff0000u));
          }
          if (t < end) {
            bf16_t *p = ys + (int64_t)t * a.y_ld;
            if constexpr (WIDE) Pack<bf16_t, 4>::store(p, v);
            else
#pragma unroll
              for (int i = 0; i < 4; ++i) p[i] = from_float<bf16_t>(v[i]);
          }
        }
      }
    }
    if (works) {
      const float decay = st.decay;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) h[nt] *= decay;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8v x = lds8(&lds.xT[wave * 16 + l16][kb * 32 + q * 8]);
        const f32x4 w0 = *(const f32x4 *)&st.weight[kb * 32 + q * 4], w1 = *(const f32x4 *)&st.weight[kb * 32 + 16 + q * 4];
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
    if (wave == 3 && t0 + kSub < end)
      steps += put_steps(lds.steps[buf ^ 1], lane, t0 + kSub + lane < end ? step_size(a, raw, bias) : 0.0f, A2);
  }
  if (PART == 1 && tid == 192 && p0 == 0) w.steps[(int64_t)slot * heads + head] = steps;
  float *h_out = PART == 1 ? w.state + ((int64_t)slot * a.channels + d) * N
                           : PART == 0 && row >= 0 && a.state_out ? a.state_out + ((int64_t)row * a.channels + d) * N : nullptr;
  if (works && h_out)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) *(f32x4 *)(h_out + nt * 16 + q * 4) = h[nt];
}

}  // namespace cortex
