// Prompts of the scan with one decay per head, as matrix products (bf16).
//
// Within a sub-chunk of 32 tokens, with c_t = sum_{s <= t} dt_s A and the state
// h that enters it,
//   y_t  = sum_{s <= t} (C_t . B_s) exp(c_t - c_s) dt_s x_s  +  exp(c_t) C_t h
//   h'   = exp(c_31) h + sum_s exp(c_31 - c_s) dt_s x_s B_s
// A workgroup takes 64 channels of one head (a wave 16 of them) and walks the
// sub-chunks of a segment with the state in its accumulators, so no state goes
// to memory between them.
//
// Precision.  x, B and C are bf16 and enter the matrix units as they are.  What
// is computed on the way (the scaled scores, the state that y reads, the
// step-weighted x that the state is summed from) is float32 and enters as three
// bf16 planes, eight bits each, which together are the value itself.  So every
// product is exact, all sums are float32, and y is rounded once, as token by token.
// (Two planes, 16 bits, would do for y's own rounding, but a y that is a small
// difference of large terms would lose it: 1e-4 of y instead of 2e-5 to 4e-5 off the
// float32 order.)  An infinite or NaN x or state makes its channel NaN from its
// token on (the token-by-token order might keep an infinity).
//
// Layouts.  A 16x16x32 product takes both operands as (index = lane & 15; 8
// consecutive k from 8 (lane >> 4)) and leaves its result as (column = lane &
// 15; rows 4 (lane >> 4) + 0..3).  The order of k is free as long as both
// operands agree: k = 8 q + 4 a + r stands for element 16 a + 4 q + r of each
// 32, of tokens as of state entries, so a result is an operand of the next
// product as it stands.  The scores are computed as B C^T (columns t), the state
// as [N, channels] and y as [channels, t].  B and x are summed over their tokens
// too: the transposing 8-byte LDS read gives a lane four rows' values of its
// column, which is the four k of one a.
//
// What it does per sub-chunk and wave at N = 128: 58 products (928 cycles of a
// SIMD's matrix unit).  The skip connection is the scores' diagonal.  Step sizes
// and their sums are made a sub-chunk ahead by one wave, beside the others'
// products.  y goes through LDS, so that z is read and y stored in whole rows.
//
// 32,768 tokens of 64 heads of 64 channels, N = 128, in segments of 2,752: 181 us
// (part 1) + 15 + 447 (part 2, 1.8 TB/s of x, z and y), traced; 538 to 568 as a
// program calls it, by the GPU.  Nothing alone bounds it: the vector unit (plane
// splits, gates: 516 instructions a wave and sub-chunk of part 2, products
// included) is busy half of the time, the matrix unit a fifth, LDS a third; the form
// with two planes took three quarters of its time without its loads and stores, or
// without its products.  12 waves a CU is what its registers allow.
#pragma once

#include "sequence.hpp"

namespace cortex {

typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4v __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2v __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kSub = 32;                 // tokens of a sub-chunk
constexpr int kHeadWaves = 4;
constexpr int kHeadThreads = 64 * kHeadWaves;

__device__ __forceinline__ f32x4 mfma_bf16x32(bf16x8v a, bf16x8v b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Position of element e in the order described above.
__device__ __forceinline__ constexpr int k_position(int e) {
  return (e & ~31) | ((e & 12) << 1) | ((e & 16) >> 2) | (e & 3);
}

// The next bf16 plane of v, two values a word: its upper halves as they are, so
// that three planes hold all of it and no finite value becomes an infinity.  v
// keeps what is left.
template <int M> __device__ __forceinline__ void plane(float (&v)[M], unsigned int (&p)[M / 2]) {
#pragma unroll
  for (int i = 0; i < M / 2; ++i) {
    const unsigned int a = __builtin_bit_cast(unsigned int, v[2 * i]), b = __builtin_bit_cast(unsigned int, v[2 * i + 1]);
    p[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    v[2 * i] -= __builtin_bit_cast(float, a & 0xffff0000u);
    v[2 * i + 1] -= __builtin_bit_cast(float, b & 0xffff0000u);
  }
}
__device__ __forceinline__ bf16x8v pack8(const unsigned int (&p)[4]) {
  return __builtin_bit_cast(bf16x8v, u32x4v{p[0], p[1], p[2], p[3]});
}

// Rows in LDS.  16-byte reads take one place of sixteen rows and the next of
// sixteen more; the hardware serves rows 0..3 and 12..15 of one place together with
// rows 4..11 of the next, and the others so.  A row of 64 elements or more is 64
// bytes longer, so that four rows start in different banks, and the places of four
// 16-byte pieces are exchanged by (- row / 4) mod 4, which keeps those sixteen
// apart.  Of an address only the lane's part is computed; sixteen rows or 32
// elements further on are constants.
template <int W> struct Rows {
  static constexpr int kStride = W >= 64 ? W + 32 : W;
  static __device__ __forceinline__ int at(int row, int pos) {
    return row * kStride + (pos & ~31) + ((((pos >> 3) ^ -(row >> 2)) & 3) << 3) + (pos & 7);
  }
};
// Rows of 64 channels, or of 64 floats: pieces exchanged by the row's number.
__device__ __forceinline__ int channel_at(int row, int ch) { return row * 64 + (((ch >> 3) ^ (row & 7)) << 3) + (ch & 7); }
__device__ __forceinline__ int float_at(int row, int ch) { return row * 64 + (((ch >> 2) ^ (row & 15)) << 2) + (ch & 3); }

// Step sizes of a sub-chunk: dt_s, c_s and what its rounding left, exp(c_s),
// exp(c_31 - c_s) dt_s, exp(c_31).
struct alignas(16) HeadSteps {
  float dt[kSub], cum[kSub], low[kSub], grow[kSub], weight[kSub], decay;
};

// Part 1 has no use for what makes y.
template <int N, bool OUTPUT> struct HeadLds {
  static constexpr int NP = N < 32 ? 32 : N;      // the products over N take 32 at a time; what is past N is 0
  typedef Rows<NP> N_;
  typedef Rows<kSub> T_;
  alignas(16) unsigned short B[kSub * N_::kStride];           // [s][n position]
  alignas(16) unsigned short C[OUTPUT ? kSub * N_::kStride : 8];           // [t][n position]
  alignas(16) unsigned short x[kSub * 64];                    // [s][channel]
  alignas(16) unsigned short M[3][OUTPUT ? kSub * T_::kStride : 8];        // scores, three planes: [t][s position]
  alignas(16) float y[OUTPUT ? kSub * 64 : 4];                             // [t][channel]
  HeadSteps steps[4];                             // of this sub-chunk, its neighbour and the next two
  float sums[kHeadWaves];
};

// A sum of two floats and what its rounding left out of it.
__device__ __forceinline__ void add_exactly(float &hi, float &lo, float b, float b_lo) {
#pragma clang fp contract(off) reassociate(off)
  const float s = hi + b, t = s - hi;
  lo = (lo + b_lo) + ((hi - (s - t)) + (b - t));
  hi = s;
}
// half_sums with the sums' roundings in `low`.
__device__ __forceinline__ float half_sums(float v, float &low) {
  low = 0.0f;
  add_exactly(v, low, shifted<0x111>(v, 0.0f), shifted<0x111>(low, 0.0f));
  add_exactly(v, low, shifted<0x112>(v, 0.0f), shifted<0x112>(low, 0.0f));
  add_exactly(v, low, shifted<0x114>(v, 0.0f), shifted<0x114>(low, 0.0f));
  add_exactly(v, low, shifted<0x118>(v, 0.0f), shifted<0x118>(low, 0.0f));
  add_exactly(v, low, shifted<0x142, 0xa>(v, 0.0f), shifted<0x142, 0xa>(low, 0.0f));
  return v;
}

// The steps of two sub-chunks, a lane a token.  The state's weights come from a sum
// from the end: those near the end, which count most, are sums of few terms.  The
// scores need sums between any two tokens, which are differences of the sums from
// the start: after one large step those are large themselves, so what their
// roundings left is kept beside them.  A step's exponent is held to -256, which
// leaves nothing of the state (the smallest float is 2^-149), so that no sum is
// infinite and no difference of two a NaN.  Returns the sum of dt over both.
__device__ __forceinline__ float put_steps(HeadSteps (&to)[4], int pair, int lane, float dt, float A2) {
#pragma clang fp contract(off)                    // each product is the same wherever it is added
  const float e = dt * A2, held = e < -256.0f ? -256.0f : e;     // (a NaN stays one)
  float low;
  const float up = half_sums(held, low);
  const float rev = __shfl_xor(dt, kSub - 1);
  const float down = half_sums(__shfl_xor(held, kSub - 1));      // from token 31 - lane of the half on
  const float after = __shfl_up(down, 1);
  const int i = lane % kSub;
  HeadSteps &st = to[2 * pair + lane / kSub];
  st.dt[i] = dt;
  st.cum[i] = up;
  st.low[i] = low;
  st.grow[i] = fast_exp2(up);
  st.weight[kSub - 1 - i] = fast_exp2(i == 0 ? 0.0f : after) * rev;
  if (i == kSub - 1) st.decay = fast_exp2(down);
  return wave_sum(dt);
}

// exp(c_t - c_s) dt_s of four tokens s.
__device__ __forceinline__ f32x4 step_scales(const HeadSteps &st, int t, int s) {
#pragma clang fp reassociate(off)
  const float ct = st.cum[t], lt = st.low[t];
  const f32x4 cs = *(const f32x4 *)&st.cum[s], ls = *(const f32x4 *)&st.low[s], dt = *(const f32x4 *)&st.dt[s];
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = fast_exp2((ct - cs[i]) + (lt - ls[i])) * dt[i];
  return r;
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

// Four elements of four rows, transposed: lane i of a group of 16 gives the address
// of row i / 4's elements 4 (i % 4) .. + 3 and gets element i of the four rows.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ s16x4 lds_columns(const unsigned short *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
__device__ __forceinline__ bf16x8v join8(s16x4 a, s16x4 b) {
  return __builtin_bit_cast(bf16x8v, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Workgroups go to the eight XCDs in turn.  Each XCD takes a run of neighbouring
// units (slot by slot, a slot's heads together), so that the heads of a group find
// its B and C in the L2 that they share.
__device__ __forceinline__ int64_t unit_of_block(int64_t units) {
  const int64_t per = (units + 7) / 8;
  return (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
}
inline unsigned blocks_of_units(int64_t units) { return (unsigned)((units + 7) / 8 * 8); }

// PART as for the channel scan: 0 whole sequences, 1 a segment's state from
// zero, 2 outputs from the state that enters it.
template <int N, int PART, bool WIDE>
__global__ void __launch_bounds__(kHeadThreads, N == 128 ? 3 : 4) head_mfma_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w, int Q,
                                                                    int64_t units) {
  typedef HeadLds<N, PART != 1> Lds;
  constexpr int NT = N / 16, NB = Lds::NP / 32;
  constexpr int OL = N / 8, kItems = (OL * kSub + kHeadThreads - 1) / kHeadThreads;   // octets of a row; of them all per thread
  __shared__ Lds lds;
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
  // Another workgroup's error may be seen by some waves and not by others.  None goes on
  // alone: the others would store what LDS held in its place.
  if (__syncthreads_or(failed != 0)) return;
  const int pw = p0 + wave * 16;                 // the wave's channels in the head
  const bool works = pw < P;                     // a head of less than 64 channels has none for the last waves
  const int d = head * P + (works ? pw : 0) + l16;

  f32x4 h[NT];                                   // rows n = 16 nt + 4 q + 0..3, column channel l16
  const float *h_in = PART == 2 ? w.state + ((int64_t)slot * a.channels + d) * N
                                : PART == 0 && row >= 0 && a.state_in ? a.state_in + ((int64_t)row * a.channels + d) * N : nullptr;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    h[nt] = works && h_in ? *(const f32x4 *)(h_in + nt * 16 + q * 4) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float A2 = decay_rate(a.A[head]), bias = a.dt_bias ? a.dt_bias[head] : 0.0f, skip = a.skip ? a.skip[head] : 0.0f;
  const bf16_t *xs = (const bf16_t *)a.x + head * P + p0, *ds = (const bf16_t *)a.dt + head;
  const bf16_t *Bs = (const bf16_t *)a.B + g * N, *Cs = (const bf16_t *)a.C + g * N;
  // the thread's eight channels of one token, of x, z and y
  const int xo = tid % 8 * 8, xt = tid / 8;
  const bool whole = p0 + xo < P;
  const int xc = whole ? xo : 0;
  const bf16_t *zs = a.z ? (const bf16_t *)a.z + head * P + p0 + xc : nullptr;
  bf16_t *ys = (bf16_t *)a.y + head * P + p0 + xc;
  float steps = 0.0f;

  // What the next sub-chunk needs, loaded while this one is worked on.  The loads
  // are unconditional, so that nothing waits for one of them: tokens past the
  // segment's end repeat its last, and are made zeros when they are stored.
  u32x4v xr, br[kItems], cr[kItems];
  const u32x4v none = {0, 0, 0, 0};
  auto fetch = [&](int t0) {
    // rows from the sub-chunk's first, in 32 bits (the host admits no longer rows)
    const int last = end - 1 - t0;
    const bool all = last >= kSub - 1;
    const bf16_t *x0 = xs + (int64_t)t0 * a.x_ld, *B0 = Bs + (int64_t)t0 * a.B_ld, *C0 = Cs + (int64_t)t0 * a.C_ld;
    const uint32_t x_ld = (uint32_t)a.x_ld, B_ld = (uint32_t)a.B_ld, C_ld = (uint32_t)a.C_ld;
    xr = load8<WIDE>(x0 + ((all ? xt : min(xt, last)) * x_ld + xc));
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid, o = id % OL * 8;
      const uint32_t s = kItems * kHeadThreads == OL * kSub && all ? id / OL : min(id / OL, min(last, kSub - 1));
      br[i] = load8<WIDE>(B0 + (s * B_ld + o));
      if (PART != 1) cr[i] = load8<WIDE>(C0 + (s * C_ld + o));
    }
  };
  // Rows of eight state entries (octet o) in k order: two halves of 8 bytes.
  auto put_row = [&](unsigned short *to, int row, int o, const u32x4v &v) {
    *(u32x2v *)(to + Lds::N_::at(row, k_position(o * 8))) = u32x2v{v[0], v[1]};
    *(u32x2v *)(to + Lds::N_::at(row, k_position(o * 8 + 4))) = u32x2v{v[2], v[3]};
  };
  if constexpr (N < 32)
    for (int i = tid; i < kSub * (Lds::NP - N) / 4; i += kHeadThreads) {
      const int s = i / ((Lds::NP - N) / 4), e = N + i % ((Lds::NP - N) / 4) * 4;
      *(u32x2v *)&lds.B[Lds::N_::at(s, k_position(e))] = u32x2v{0, 0};
      if (PART != 1) *(u32x2v *)&lds.C[Lds::N_::at(s, k_position(e))] = u32x2v{0, 0};
    }
  // the tile above the diagonal, which a product over 32 tokens reaches
  if (PART != 1 && wave < 3)
    *(u32x2v *)&lds.M[wave][Lds::T_::at(l16, k_position(16 + q * 4))] = u32x2v{0, 0};

  // Steps are made two sub-chunks ahead for two of them, by the waves in turn.
  auto raw_step = [&](int t0) { return to_float<bf16_t>(ds[(int64_t)min(t0 + lane, end - 1) * a.dt_ld]); };
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
    // Everyone is done with the last sub-chunk's B, C, x and scores: they are read
    // before its y is exchanged.
    if (PART == 1) __syncthreads();
    if (t0 + kSub > end) {
      if (t0 + xt >= end) xr = none;
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        if (t0 + (i * kHeadThreads + tid) / OL >= end) br[i] = cr[i] = none;
    }
    *(u32x4v *)&lds.x[channel_at(xt, xo)] = xr;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kHeadThreads + tid, s = id / OL;
      if (kItems * kHeadThreads == OL * kSub || s < kSub) {
        put_row(lds.B, s, id % OL, br[i]);
        if (PART != 1) put_row(lds.C, s, id % OL, cr[i]);
      }
    }
    __syncthreads();
    if (t0 + kSub < end) fetch(t0 + kSub);
    const float raw = makes ? raw_step(t0 + 2 * kSub) : 0.0f;
    const HeadSteps &st = lds.steps[k % 4];
    // x of the wave's channels, over the tokens
    const bf16x8v x = join8(lds_columns(&lds.x[channel_at(q * 4 + l16 / 4, wave * 16 + l16 % 4 * 4)]),
                            lds_columns(&lds.x[channel_at(16 + q * 4 + l16 / 4, wave * 16 + l16 % 4 * 4)]));
    u32x4v zr = none;
    f32x4 y[2];
    if constexpr (PART != 1) {
      if (zs) zr = load8<WIDE>(zs + (int64_t)t0 * a.z_ld + min(xt, end - 1 - t0) * (uint32_t)a.z_ld);
      // Scores: the tiles (0,0) (1,0) (1,1) on and below the diagonal, one a wave.
      if (wave < 3) {
        const int ti = wave > 0, si = wave > 1;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int m = 0; m < NB; ++m)
          acc = mfma_bf16x32(lds8(&lds.B[Lds::N_::at(si * 16 + l16, m * 32 + q * 8)]),
                             lds8(&lds.C[Lds::N_::at(ti * 16 + l16, m * 32 + q * 8)]), acc);
        const int t = ti * 16 + l16, s = si * 16 + q * 4;
        const f32x4 scale = step_scales(st, t, s);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = s + i <= t ? acc[i] * scale[i] : 0.0f;
          if (s + i == t) v[i] += skip;
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          unsigned int b[2];
          plane(v, b);
          *(u32x2v *)&lds.M[p][Lds::T_::at(t, k_position(s))] = u32x2v{b[0], b[1]};
        }
      }
      // From the state: rows channels, columns t.
      y[0] = y[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (works) {
#pragma unroll
        for (int m = 0; m < NB; ++m) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = h[2 * m][i];
            v[4 + i] = 2 * m + 1 < NT ? h[2 * m + 1 < NT ? 2 * m + 1 : 0][i] : 0.0f;
          }
          unsigned int b[4];
          plane(v, b);
          const bf16x8v h0 = pack8(b);
          plane(v, b);
          const bf16x8v h1 = pack8(b);
          plane(v, b);
          const bf16x8v h2 = pack8(b);
#pragma unroll
          for (int ti = 0; ti < 2; ++ti) {
            const bf16x8v c = lds8(&lds.C[Lds::N_::at(ti * 16 + l16, m * 32 + q * 8)]);
            y[ti] = mfma_bf16x32(h2, c, y[ti]);
            y[ti] = mfma_bf16x32(h1, c, y[ti]);
            y[ti] = mfma_bf16x32(h0, c, y[ti]);
          }
        }
#pragma unroll
        for (int ti = 0; ti < 2; ++ti) y[ti] *= st.grow[ti * 16 + l16];
      }
    }
    // The state's update.
    if (works) {
      const float decay = st.decay;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) h[nt] *= decay;
      const f32x4 w0 = *(const f32x4 *)&st.weight[q * 4], w1 = *(const f32x4 *)&st.weight[16 + q * 4];
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = (float)x[i] * w0[i];
        v[4 + i] = (float)x[4 + i] * w1[i];
      }
      unsigned int b[4];
      plane(v, b);
      const bf16x8v x0 = pack8(b);
      plane(v, b);
      const bf16x8v x1 = pack8(b);
      plane(v, b);
      const bf16x8v x2 = pack8(b);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int n = k_position(nt * 16 + l16 % 4 * 4);
        const bf16x8v bt = join8(lds_columns(&lds.B[Lds::N_::at(q * 4 + l16 / 4, n)]),
                                 lds_columns(&lds.B[Lds::N_::at(16 + q * 4 + l16 / 4, n)]));
        h[nt] = mfma_bf16x32(bt, x2, h[nt]);
        h[nt] = mfma_bf16x32(bt, x1, h[nt]);
        h[nt] = mfma_bf16x32(bt, x0, h[nt]);
      }
    }
    if (makes) make_steps(t0 + 2 * kSub, (k / 2 + 1) % 2, raw);
    if constexpr (PART != 1) {
      __syncthreads();                           // the scores are there
      if (works) {
        // The products with the zeros above the diagonal would carry an infinite or NaN x (an
        // exponent of all ones) to the tokens before it.  It is left out of them, and its
        // channel's tokens from its own on become NaN.
        const u32x4v bits = __builtin_bit_cast(u32x4v, x);
        bf16x8v xf = x;
        unsigned int odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= ((bits[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        const bool any_odd = __any(odd != 0);
        int first = kSub;
        if (any_odd) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float v = (float)x[j];
            if (!(__builtin_fabsf(v) < __builtin_inff())) {
              const int s = (j < 4 ? 0 : 12) + q * 4 + j;
              first = s < first ? s : first;
              xf[j] = (__bf16)0.0f;
            }
          }
          first = min(first, __shfl_xor(first, 16));
          first = min(first, __shfl_xor(first, 32));
        }
#pragma unroll
        for (int p = 2; p >= 0; --p)
#pragma unroll
          for (int ti = 0; ti < 2; ++ti)
            y[ti] = mfma_bf16x32(xf, lds8(&lds.M[p][Lds::T_::at(ti * 16 + l16, q * 8)]), y[ti]);
        if (any_odd)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int from = __shfl(first, q * 4 + i);
#pragma unroll
            for (int ti = 0; ti < 2; ++ti)
              if (ti * 16 + l16 >= from) y[ti][i] = __builtin_nanf("");
          }
#pragma unroll
        for (int ti = 0; ti < 2; ++ti) *(f32x4 *)&lds.y[float_at(ti * 16 + l16, wave * 16 + q * 4)] = y[ti];
      }
      __syncthreads();                           // y is there
      if (whole && t0 + xt < end) {
        const f32x4 lo = *(const f32x4 *)&lds.y[float_at(xt, xo)];
        const f32x4 hi = *(const f32x4 *)&lds.y[float_at(xt, xo + 4)];
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (zs)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] *= silu(__builtin_bit_cast(float, zr[i] << 16));
            v[2 * i + 1] *= silu(__builtin_bit_cast(float, zr[i] & 0xffff0000u));
          }
        bf16_t *p = ys + (int64_t)t0 * a.y_ld + xt * (uint32_t)a.y_ld;
        if constexpr (WIDE) Pack<bf16_t, 8>::store(p, v);
        else
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = from_float<bf16_t>(v[i]);
      }
    }
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
