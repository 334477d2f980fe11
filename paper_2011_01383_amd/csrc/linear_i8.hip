// Rows to 8 bits, and the projection that multiplies them.
//
// Weights are the first operand of the matrix units and tokens the second, so a
// lane ends with four neighbouring channels of one token.  Sums are whole numbers in 32
// bits, which are exact, so no order of them and no split changes a result.
#include "sequence.hpp"

namespace cortex {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int64_t kMaxRow = 1 << 24;              // 255 rows of bytes stay below 2^32
constexpr int32_t kMaxInputs = 131071;           // 128 * 128 of each stay below 2^31
// A grid has less than 2^32 threads: up to 1,024 to a row that is brought to 8 bits, 512 to 16 channels of few tokens, 1,024 to a
// tile of 256 by 256.
constexpr int32_t kMaxRows = 1 << 22;
constexpr int32_t kMaxOutputs = 1 << 26;
constexpr int64_t kMaxResults = (int64_t)1 << 37;

// ---------------------------------------------------------------------------
// Rows to 8 bits
// ---------------------------------------------------------------------------
// The scale of a row whose largest |x| has the bits of `top`.
struct RowScale {
  float scale;
  bool none;                                     // its values are all 0
  float lift, lifted, inverse;                   // 2^64 for small rows, else 1; scale times it; the reciprocal of that
  __device__ __forceinline__ explicit RowScale(unsigned int top) {
    const bool odd = top >= 0x7f800000u;         // infinities and NaN are the largest
    scale = odd ? __builtin_nanf("") : __builtin_bit_cast(float, top) / 127.0f;
    none = odd || scale == 0.0f;
    lift = scale < 0x1p-64f ? 0x1p64f : 1.0f;
    lifted = scale * lift;
    inverse = 1.0f / lifted;
  }
};

// Eight elements; `n` of them are there, the others 0.
template <typename T, bool WIDE> __device__ __forceinline__ void load_eight(const T *x, int n, float (&v)[8]) {
  if (WIDE) {
    if (n > 0) {
      Pack<T, 8>::load(x, v);
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_float<T>(x[i]) : 0.0f;
  }
}

// x / scale rounded to a whole number.  With the reciprocal rounded correctly, a quotient off by less than a step becomes
// the correctly rounded one by one step of q + (x - q scale) / scale, whose remainder is exact (Markstein 1990); q = x / scale as
// a product may be off by two, so there are two such steps.  Small rows are lifted by a power of two, which changes no
// quotient, so that remainders do not underflow; a scale in the denormals may leave a quotient above 127.  The sum with 1.5 2^23
// rounds to whole numbers, which then are its low bits.  Divisions took most of the time: 8,192 rows of 4,096 28 us.
__device__ __forceinline__ u32x2 quant_eight(const float (&v)[8], const RowScale &s) {
#pragma clang fp contract(off) reassociate(off)
  unsigned int b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i] * s.lift;
    float q = x * s.inverse;
    q = __builtin_fmaf(__builtin_fmaf(-q, s.lifted, x), s.inverse, q);
    q = __builtin_fmaf(__builtin_fmaf(-q, s.lifted, x), s.inverse, q);
    b[i] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_fmed3f(q, -127.0f, 127.0f) + 12582912.0f);
  }
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    r[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u), 0x05040100u);
  return s.none ? u32x2{0u, 0u} : r;
}

// |x| as whole numbers keep their order.
__device__ __forceinline__ unsigned int top_of(const float (&v)[8], unsigned int top) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(unsigned int, v[i]) & 0x7fffffffu);
  return top;
}
__device__ __forceinline__ unsigned int wave_top(unsigned int top) {
#pragma unroll
  for (int m = 32; m; m >>= 1) top = max(top, (unsigned int)__shfl_xor((int)top, m));
  return top;
}

// A workgroup of THREADS a row, which it keeps in registers (KEPT: 16 elements a thread), or, where it has more columns, reads
// again from the caches.  `filled`: columns of q that are written, zeros past the row's own.  WIDE: rows of x and q in
// whole eights at their alignment.  The bytes bound it: 8,192 rows of 4,096 bf16 take 21 us, 4.7 TB/s.
template <typename T, bool WIDE, int THREADS, bool KEPT>
__global__ void __launch_bounds__(THREADS) quant_kernel(cortex_quant_i8_t a, int32_t *status, int filled) {
  constexpr int kWaves = THREADS / 64, kStride = THREADS * 8, kKeep = KEPT ? 2 : 1;
  __shared__ unsigned int most[kWaves];
  if (__syncthreads_or(entry_status(status) != 0)) return;
  const int tid = (int)threadIdx.x;
  const int64_t r = blockIdx.x;
  const T *x = (const T *)a.x + r * a.x_ld;
  int8_t *q = a.q + r * a.q_ld;
  float v[kKeep][8];
  unsigned int top = 0;
  if constexpr (KEPT) {
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
      const int c = tid * 8 + k * kStride;
      load_eight<T, WIDE>(x + c, a.columns - c, v[k]);
    }
#pragma unroll
    for (int k = 0; k < kKeep; ++k) top = top_of(v[k], top);
  } else {
    for (int c = tid * 8; c < a.columns; c += kStride) {
      load_eight<T, WIDE>(x + c, a.columns - c, v[0]);
      top = top_of(v[0], top);
    }
  }
  top = wave_top(top);
  if ((tid & 63) == 0) most[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = max(top, most[w]);
  const RowScale s(__builtin_amdgcn_readfirstlane(top));
  auto put = [&](int c, const float (&u)[8]) {
    if (c >= filled) return;
    const u32x2 b = quant_eight(u, s);
    if (WIDE) {
      *(u32x2 *)(q + c) = b;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < filled) q[c + i] = (int8_t)(b[i / 4] >> (8 * (i % 4)));
    }
  };
  if constexpr (KEPT) {
#pragma unroll
    for (int k = 0; k < kKeep; ++k) put(tid * 8 + k * kStride, v[k]);
  } else {
    for (int c = tid * 8; c < filled; c += kStride) {
      load_eight<T, WIDE>(x + c, a.columns - c, v[0]);
      put(c, v[0]);
    }
  }
  if (tid == 0) a.scale[r] = s.scale;
}

template <typename T, bool WIDE, int THREADS, bool KEPT> void launch_quant_of(const cortex_quant_i8_t &a, int32_t *status, int filled, hipStream_t st) {
  quant_kernel<T, WIDE, THREADS, KEPT><<<(unsigned)a.rows, THREADS, 0, st>>>(a, status, filled);
}

template <typename T, bool WIDE> int launch_quant_rows(const cortex_quant_i8_t &a, int32_t *status, int filled, void *stream) {
  const hipStream_t st = (hipStream_t)stream;
  // As few waves as hold a row: 8,192 rows of 1,000 (with a product over 64 channels) by one wave 13.8 us, two 19, four 22.6; of 2,048
  // by two 20.5, four 29.7; of 4,096 by four 34.3, two (32 elements a thread) 37.1; of 8,192
  // by eight 73, read again by four 76 (float32 93 and 118); 7 rows of 6,098 10.6 and 13.2; 1,024 float32 rows of 16,384 by sixteen 51,
  // read again by four 58.
  if (filled <= 1024) launch_quant_of<T, WIDE, 64, true>(a, status, filled, st);
  else if (filled <= 2048) launch_quant_of<T, WIDE, 128, true>(a, status, filled, st);
  else if (filled <= 4096) launch_quant_of<T, WIDE, 256, true>(a, status, filled, st);
  else if (filled <= 8192) launch_quant_of<T, WIDE, 512, true>(a, status, filled, st);
  else if (filled <= 16384) launch_quant_of<T, WIDE, 1024, true>(a, status, filled, st);
  else launch_quant_of<T, WIDE, 1024, false>(a, status, filled, st);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T> bool eights(const void *x, int64_t x_ld, int columns) {
  return columns % 8 == 0 && x_ld % 8 == 0 && ((uintptr_t)x & (8 * sizeof(T) - 1)) == 0;
}

template <typename T> int launch_quant(const cortex_quant_i8_t &a, int32_t *status, int filled, void *stream) {
  const bool wide = eights<T>(a.x, a.x_ld, a.columns) && filled % 8 == 0 && a.q_ld % 8 == 0 && ((uintptr_t)a.q & 7) == 0;
  return wide ? launch_quant_rows<T, true>(a, status, filled, stream) : launch_quant_rows<T, false>(a, status, filled, stream);
}

// 8-bit rows of any alignment into rows of whole pieces, zeros at their ends.
__global__ void __launch_bounds__(256) pad_kernel(const int8_t *x, int64_t x_ld, int columns, int8_t *to, int64_t to_ld,
                                                  int32_t *status) {
  if (entry_status(status) != 0) return;
  const int64_t r = blockIdx.x;
  for (int c = (int)threadIdx.x; c < to_ld; c += 256) to[r * to_ld + c] = c < columns ? x[r * x_ld + c] : (int8_t)0;
}

// ---------------------------------------------------------------------------
// The product
// ---------------------------------------------------------------------------
constexpr int kDepth = 64;                       // bytes of the inputs at a time

// What a product kernel takes: x in rows of a multiple of kDepth bytes, zeros past the
// inputs, so that what w holds there does not matter; `pieces` of 16 bytes of a row of w are read.
struct Product {
  const int8_t *x, *w;
  int64_t x_ld, w_ld, y_ld;
  const float *x_scale, *w_scale, *bias;
  void *y;
  int32_t tokens, outputs, pieces;
};

// Scales and biases of four neighbouring channels from n on.
struct Four {
  float scale[4], bias[4];
  __device__ __forceinline__ void load(const Product &a, int n) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at = min(n + r, a.outputs - 1);
      scale[r] = a.w_scale[at];
      bias[r] = a.bias ? a.bias[at] : 0.0f;
    }
  }
};

template <typename T> __device__ __forceinline__ T finish(const Product &a, int acc, float xs, float ws, float bias) {
#pragma clang fp contract(off)
  float v = (float)acc * xs * ws;
  if (a.bias) v += bias;
  return from_float<T>(v);
}

// Four neighbouring channels of one token.
template <typename T> __device__ __forceinline__ void put_four(const Product &a, i32x4 acc, float xs, const Four &f, int t, int n, bool aligned) {
  T *y = (T *)a.y + (int64_t)t * a.y_ld;
  if (aligned && n + 3 < a.outputs) {
    typedef T pack __attribute__((ext_vector_type(4)));
    pack v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = finish<T>(a, acc[r], xs, f.scale[r], f.bias[r]);
    *(pack *)(y + n) = v;
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < a.outputs) y[n + r] = finish<T>(a, acc[r], xs, f.scale[r], f.bias[r]);
  }
}

// A row of 64 bytes in LDS, its four 16-byte pieces exchanged so that the rows and pieces
// that the hardware serves together (rows 0-3 and 12-15 of sixteen with rows 4-11 of
// the next piece) lie in different banks.
__device__ __forceinline__ int piece_place(int row, int piece) { return piece ^ (-(row >> 2) & 3); }

// Tiles of TN channels and TT tokens by WN x WT waves; BUFFERS stages of kDepth bytes in
// LDS, all but one of them on their way while one is multiplied.  XCDs take runs of
// neighbouring tiles, four tiles of tokens by as many of channels as there are.
//
// 8,192 tokens, 4,096 inputs, 8,192 channels in tiles of 256 by 256: 258 us (252 to 262 in five runs), 2.13e15 operations a
// second, the matrix units busy 55% of it, no conflicts in LDS.  Sixteen waves of 64 by 64 (4 a SIMD) and four buffers; in its place eight waves 331,
// four of 128 by 128 470, three buffers 329, two of 128 bytes 317, tiles of 128 by 128 391, all with the rows' 28, of a
// form that took 303 in all.
template <typename T, int TN, int TT, int WN, int WT, int BUFFERS>
__global__ void __launch_bounds__(64 * WN * WT) product_kernel(Product a, const int32_t *status, bool aligned, int n_tiles, int t_tiles) {
  constexpr int kWaves = WN * WT, I = TN / WN / 16, J = TT / WT / 16, kStage = (TN + TT) * kDepth;
  constexpr int kCopies = (TN + TT) / 16 / kWaves;         // of 16 rows each, per wave and stage
  // Scales and biases come first: the last stage does not wait for them then.  They stay in registers
  // where there are some, else in LDS.
  constexpr bool kEarly = kWaves <= 4;
  __shared__ __attribute__((aligned(1024))) int8_t lds[BUFFERS * kStage];
  __shared__ __attribute__((aligned(16))) float late[kEarly ? 1 : 2 * TN + TT];
  const int64_t total = (int64_t)n_tiles * t_tiles, tile = unit_of_block(total);
  if (tile >= total) return;
  if (__syncthreads_or(entry_status(status) != 0)) return;
  const int lane = (int)threadIdx.x & 63, q = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int band = (int)(tile / (4 * n_tiles)), rest = (int)(tile % (4 * n_tiles)), tall = min(4, t_tiles - band * 4);
  const int n0 = rest / tall * TN, t0 = (band * 4 + rest % tall) * TT;
  const int wn = wave % WN * (TN / WN), wt = wave / WN * (TT / WT);
  const int8_t *ws = a.w + (int64_t)n0 * a.w_ld, *xs = a.x + (int64_t)t0 * a.x_ld;
  const uint32_t lds0 = lds_place(lds);
  // The lane's piece of each copy; a copy is of w or of x alone.
  uint32_t offset[kCopies];
  int piece[kCopies];
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {
    const int row = (wave * kCopies + i) * 16 + lane / 4;
    piece[i] = piece_place(row, lane % 4);
    offset[i] = row < TN ? (uint32_t)min(row, a.outputs - 1 - n0) * (uint32_t)a.w_ld
                         : (uint32_t)min(row - TN, a.tokens - 1 - t0) * (uint32_t)a.x_ld;
  }
  const int steps = (a.pieces + 3) / 4;
  auto copy = [&](int step, int buffer) {
    step = min(step, steps - 1);                 // past the end: once more the last, so that the count of copies on their way is fixed
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int first = (wave * kCopies + i) * 16;
      const bool of_w = first < TN;
      // what w lacks of the last stage repeats its last piece
      const uint32_t p = of_w ? (uint32_t)min(step * 4 + piece[i], a.pieces - 1) : (uint32_t)(step * 4 + piece[i]);
      copy_to_lds(of_w ? ws : xs, offset[i] + p * 16, lds0 + (uint32_t)(buffer * kStage + first * kDepth));
    }
  };
  i32x4 acc[I][J];
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  Four four[I];
  float xscale[J];
  if constexpr (kEarly) {
#pragma unroll
    for (int i = 0; i < I; ++i) four[i].load(a, n0 + wn + i * 16 + q * 4);
#pragma unroll
    for (int j = 0; j < J; ++j) xscale[j] = a.x_scale[min(t0 + wt + j * 16 + l16, a.tokens - 1)];
  } else {
    static_assert(2 * TN + TT <= 64 * kWaves, "a thread each");
    const int c = (int)threadIdx.x;
    if (c < TN) late[c] = a.w_scale[min(n0 + c, a.outputs - 1)];
    else if (c < 2 * TN) late[c] = a.bias ? a.bias[min(n0 + c - TN, a.outputs - 1)] : 0.0f;
    else if (c < 2 * TN + TT) late[c] = a.x_scale[min(t0 + c - 2 * TN, a.tokens - 1)];
  }
#pragma unroll
  for (int b = 0; b < BUFFERS - 1; ++b) copy(b, b);
  i32x4 wf[2][I], xf[2][J];
  auto read = [&](int buffer, i32x4 (&wr)[I], i32x4 (&xr)[J]) {
    const int8_t *w = lds + buffer * kStage, *x = w + TN * kDepth;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int row = wn + i * 16 + l16;
      wr[i] = *(const i32x4 *)(w + row * kDepth + piece_place(row, q) * 16);
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int row = wt + j * 16 + l16;
      xr[j] = *(const i32x4 *)(x + row * kDepth + piece_place(row, q) * 16);
    }
  };
  copies_done<(BUFFERS - 2) * kCopies>();
  __syncthreads();
  read(0, wf[0], xf[0]);
  int buffer = 0;
  // One stage is multiplied from registers while the next is read from LDS.
  auto multiply = [&](int step, const i32x4 (&wc)[I], const i32x4 (&xc)[J], i32x4 (&wr)[I], i32x4 (&xr)[J]) {
    copies_done<(BUFFERS - 3) * kCopies>();
    __syncthreads();                             // the next stage is there, the one before this is multiplied
    copy(step + BUFFERS - 1, buffer == 0 ? BUFFERS - 1 : buffer - 1);
    buffer = buffer == BUFFERS - 1 ? 0 : buffer + 1;
    read(buffer, wr, xr);
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wc[i], xc[j], acc[i][j], 0, 0, 0);
  };
#pragma unroll 1
  for (int step = 0; step < steps; step += 2) {
    multiply(step, wf[0], xf[0], wf[1], xf[1]);
    if (step + 1 < steps) multiply(step + 1, wf[1], xf[1], wf[0], xf[0]);
  }
  copies_done<0>();                              // LDS is given back only when nothing is on its way to it
  if constexpr (!kEarly) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const f32x4 s = *(const f32x4 *)&late[wn + i * 16 + q * 4], b = *(const f32x4 *)&late[TN + wn + i * 16 + q * 4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        four[i].scale[r] = s[r];
        four[i].bias[r] = b[r];
      }
    }
#pragma unroll
    for (int j = 0; j < J; ++j) xscale[j] = late[2 * TN + wt + j * 16 + l16];
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int t = t0 + wt + j * 16 + l16;
    if (t >= a.tokens) continue;
#pragma unroll
    for (int i = 0; i < I; ++i) put_four<T>(a, acc[i][j], xscale[j], four[i], t, n0 + wn + i * 16 + q * 4, aligned);
  }
}

// Few tokens: a workgroup has 16 TI channels and all tokens (16 TJ of them at most), its
// waves every WAVES-th 64 bytes of the inputs; operands go to registers, AHEAD of the
// wave's shares at once.  The weights' bytes bound it, and the latency of one workgroup: 64 tokens, 2,048 inputs, 8,192
// channels (16.8 MB) take 9.5 us.
template <typename T, int TI, int TJ, int WAVES, int AHEAD>
__global__ void __launch_bounds__(64 * WAVES) few_kernel(Product a, const int32_t *status, bool aligned) {
  __shared__ i32x4 sums[WAVES][TI * TJ][64];
  const int failed = entry_status(status);
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, q = lane >> 4, l16 = lane & 15;
  const int n0 = (int)blockIdx.x * 16 * TI;
  const int8_t *w[TI], *x[TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i) w[i] = a.w + (int64_t)min(n0 + i * 16 + l16, a.outputs - 1) * a.w_ld;
#pragma unroll
  for (int j = 0; j < TJ; ++j) x[j] = a.x + (int64_t)min(j * 16 + l16, a.tokens - 1) * a.x_ld;
  const int steps = (a.pieces + 3) / 4;          // of 64 bytes
  // the wave's tile of the results, and what it is multiplied by
  static_assert(TI * TJ <= WAVES, "a tile a wave");
  const int t = wave % TJ * 16 + l16, n = n0 + wave / TJ * 16 + q * 4;
  Four four;
  four.load(a, n);
  const float xscale = a.x_scale[min(t, a.tokens - 1)];
  i32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll 1
  for (int s0 = wave; s0 < steps; s0 += WAVES * AHEAD) {
    i32x4 wf[AHEAD][TI], xf[AHEAD][TJ];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      // what lies past the end is multiplied by x's zeros, or not at all
      const int p = min(s0 + k * WAVES, steps - 1) * 4 + q;
#pragma unroll
      for (int i = 0; i < TI; ++i) wf[k][i] = *(const i32x4 *)(w[i] + (int64_t)min(p, a.pieces - 1) * 16);
#pragma unroll
      for (int j = 0; j < TJ; ++j) xf[k][j] = *(const i32x4 *)(x[j] + (int64_t)p * 16);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (s0 + k * WAVES < steps)
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
          for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[k][i], xf[k][j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) sums[wave][i * TJ + j][lane] = acc[i][j];
  if (__syncthreads_or(failed != 0)) return;
  if (wave >= TI * TJ || t >= a.tokens) return;
  i32x4 s = sums[0][wave][lane];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) s += sums[i][wave][lane];
  put_four<T>(a, s, xscale, four, t, n, aligned);
}

// One token, brought to 8 bits by every workgroup for itself, beside the loads of its first
// weights: a launch less.  The row stays in LDS.  4,096 inputs by 8,192 channels 9.4 us, 3.6 TB/s of weights.
constexpr int kOwnBytes = 16384;
template <typename T, bool WIDE, int WAVES, int AHEAD>
__global__ void __launch_bounds__(64 * WAVES) own_kernel(Product a, const T *x, int columns, const int32_t *status, bool aligned) {
  constexpr int kThreads = 64 * WAVES;
  __shared__ __attribute__((aligned(16))) int8_t row[kOwnBytes];
  __shared__ i32x4 sums[WAVES][64];
  __shared__ unsigned int most[WAVES];
  const int failed = entry_status(status);
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4, l16 = lane & 15;
  const int n0 = (int)blockIdx.x * 16, steps = (a.pieces + 3) / 4;
  const int8_t *w = a.w + (int64_t)min(n0 + l16, a.outputs - 1) * a.w_ld;
  i32x4 wf[AHEAD];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      wf[k] = *(const i32x4 *)(w + (int64_t)min(min(s0 + k * WAVES, steps - 1) * 4 + q, a.pieces - 1) * 16);
  };
  // Most of the row stays in registers until its scale is known.
  constexpr int kKeep = 2;
  float v[kKeep][8];
#pragma unroll
  for (int k = 0; k < kKeep; ++k) {
    const int c = (k * kThreads + tid) * 8;
    load_eight<T, WIDE>(x + c, columns - c, v[k]);
  }
  fetch(wave);
  Four four;
  four.load(a, n0 + q * 4);
  unsigned int top = 0;
#pragma unroll
  for (int k = 0; k < kKeep; ++k) top = top_of(v[k], top);
  for (int c = (kKeep * kThreads + tid) * 8; c < columns; c += kThreads * 8) {
    float u[8];
    load_eight<T, WIDE>(x + c, columns - c, u);
    top = top_of(u, top);
  }
  top = wave_top(top);
  if (lane == 0) most[wave] = top;
  if (__syncthreads_or(failed != 0)) return;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) top = max(top, most[i]);
  const RowScale s(__builtin_amdgcn_readfirstlane(top));
#pragma unroll
  for (int k = 0; k < kKeep; ++k) {
    const int c = (k * kThreads + tid) * 8;
    if (c < steps * 64) *(u32x2 *)&row[c] = quant_eight(v[k], s);
  }
  for (int c = (kKeep * kThreads + tid) * 8; c < steps * 64; c += kThreads * 8) {
    float u[8];
    load_eight<T, WIDE>(x + c, columns - c, u);
    *(u32x2 *)&row[c] = quant_eight(u, s);
  }
  __syncthreads();
  i32x4 acc = {0, 0, 0, 0};
#pragma unroll 1
  for (int s0 = wave; s0 < steps; s0 += WAVES * AHEAD) {
    if (s0 != wave) fetch(s0);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (s0 + k * WAVES < steps)
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[k], *(const i32x4 *)(row + (s0 + k * WAVES) * 64 + q * 16), acc, 0, 0, 0);
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || l16 != 0) return;
#pragma unroll
  for (int i = 1; i < WAVES; ++i) acc += sums[i][lane];
  put_four<T>(a, acc, s.scale, four, 0, n0 + q * 4, aligned);
}

// ---------------------------------------------------------------------------
// The call
// ---------------------------------------------------------------------------
// The workspace: tokens in 8 bits, in rows of whole stages, and their scales.
static int64_t row_bytes(int32_t inputs) { return ((int64_t)inputs + kDepth - 1) / kDepth * kDepth; }
static size_t linear_bytes(int64_t tokens, int32_t inputs) {
  return align_up((size_t)(tokens * row_bytes(inputs)), 256) + align_up((size_t)tokens * 4, 256);
}

static bool bad_linear_size(int32_t tokens, int32_t outputs, int32_t inputs) {
  return tokens < 0 || outputs < 1 || outputs > kMaxOutputs || (int64_t)tokens * outputs > kMaxResults || inputs < 1 ||
         inputs > kMaxInputs;
}

template <typename T, int TN, int TT, int WN, int WT, int BUFFERS>
int launch_tiles(const Product &p, const int32_t *status, bool aligned, hipStream_t st) {
  const int n_tiles = (p.outputs + TN - 1) / TN, t_tiles = (p.tokens + TT - 1) / TT;
  product_kernel<T, TN, TT, WN, WT, BUFFERS>
      <<<blocks_of_units((int64_t)n_tiles * t_tiles), 64 * WN * WT, 0, st>>>(p, status, aligned, n_tiles, t_tiles);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T, int TI, int TJ, int WAVES>
int launch_few(const Product &p, const int32_t *status, bool aligned, hipStream_t st) {
  const unsigned grid = (unsigned)((p.outputs + 16 * TI - 1) / (16 * TI));
  // No more loads at once than a wave has shares, or it loads the last one again: 10,000 channels of 500 inputs, 64
  // tokens 9.2 us and 14.9, 7 tokens 7.0 and 10.0.
  const int each = ((p.pieces + 3) / 4 + WAVES - 1) / WAVES;
  if (each <= 1) few_kernel<T, TI, TJ, WAVES, 1><<<grid, 64 * WAVES, 0, st>>>(p, status, aligned);
  else if (each <= 2) few_kernel<T, TI, TJ, WAVES, 2><<<grid, 64 * WAVES, 0, st>>>(p, status, aligned);
  else few_kernel<T, TI, TJ, WAVES, 4><<<grid, 64 * WAVES, 0, st>>>(p, status, aligned);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T> int launch_product(const Product &p, const int32_t *status, bool aligned, hipStream_t st) {
  // Up to 64 tokens against tiles of 64 by 64, over 2,048 inputs: 16 tokens of 1,024 channels 9.3 us and 11.4, 64 of 8,192
  // 13.4 and 14.2.
  if (p.tokens <= 64) {
    // Four, eight and sixteen waves: 7 tokens, 2,695 channels of 8,140 inputs, 19.5 us, 17.5 and 17.6, 10,000 of 500 6.8, 7.0
    // and 7.9.
    if (p.tokens <= 16) return launch_few<T, 1, 1, 8>(p, status, aligned, st);
    // 32 channels a workgroup where that leaves one a CU, else 16 (2,048 inputs): 24 tokens of 4,096 channels 10.0 us and 8.4, of
    // 8,192 10.7 and 11.9; 64 tokens of 4,096 12.8 and 11.5, of 8,192 13.3 and 16.4.
    const bool many = (p.outputs + 15) / 16 >= 512;
    if (p.tokens <= 32) return many ? launch_few<T, 2, 2, 8>(p, status, aligned, st) : launch_few<T, 1, 2, 8>(p, status, aligned, st);
    return many ? launch_few<T, 2, 4, 8>(p, status, aligned, st) : launch_few<T, 1, 4, 8>(p, status, aligned, st);
  }
  // The largest tiles that keep three of four CUs at work, over 2,048 inputs in tiles of 256, 128 and 64: 128 tokens of
  // 2,048 channels 35.9, 25.6 and 13.0 us, 1,024 of 2,048 43.8, 28.9 and 20.0, 1,024 of 8,192 48.2, 42.9 and 57.1, 2,048 of
  // 8,192 54, 75 and 106, 4,096 of 8,192 105, 146 and 210.
  auto tiles = [&](int64_t n, int64_t t) { return (p.outputs + n - 1) / n * ((p.tokens + t - 1) / t); };
  if (tiles(256, 256) >= 192) return launch_tiles<T, 256, 256, 4, 4, 4>(p, status, aligned, st);
  if (tiles(128, 128) >= 192) return launch_tiles<T, 128, 128, 2, 2, 4>(p, status, aligned, st);
  return launch_tiles<T, 64, 64, 2, 2, 8>(p, status, aligned, st);
}

template <typename T, bool WIDE> int launch_own(const Product &p, int inputs, const int32_t *status, bool aligned, hipStream_t st) {
  const unsigned grid = (unsigned)((p.outputs + 15) / 16);
  const T *x = (const T *)p.x;
  const int shares = (p.pieces + 3) / 4;
  // Eight waves where that leaves each eight shares of the weights, all loaded at once, else four, and no more loads than shares: 8,192
  // channels of 4,096 inputs by eight waves 9.4 us, by four 10.1, 4,096 of 8,192 10.0 and 12.7, but 8,192 of 2,048 7.6 and 6.6;
  // 10,000 of 500 by two loads at once 5.4 and by eight 6.9.
  if (shares >= 64) own_kernel<T, WIDE, 8, 8><<<grid, 512, 0, st>>>(p, x, inputs, status, aligned);
  else if (shares > 16) own_kernel<T, WIDE, 4, 8><<<grid, 256, 0, st>>>(p, x, inputs, status, aligned);
  else if (shares > 8) own_kernel<T, WIDE, 4, 4><<<grid, 256, 0, st>>>(p, x, inputs, status, aligned);
  else own_kernel<T, WIDE, 4, 2><<<grid, 256, 0, st>>>(p, x, inputs, status, aligned);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T> int launch_linear(const cortex_linear_i8_t &a, int32_t *status, void *ws, void *stream) {
  const hipStream_t st = (hipStream_t)stream;
  const int64_t row = row_bytes(a.inputs);
  Product p = {(const int8_t *)a.x, a.w, a.x_ld, a.w_ld, a.y_ld, a.x_scale, a.w_scale, a.bias, a.y, a.tokens, a.outputs, (a.inputs + 15) / 16};
  int8_t *rows = (int8_t *)ws;
  float *scales = (float *)(rows + align_up((size_t)(a.tokens * row), 256));
  const bool aligned = a.y_ld % 4 == 0 && ((uintptr_t)a.y & (4 * sizeof(T) - 1)) == 0;
  // One token in one launch against two: 300 channels of 300 inputs 3.8 us and 5.6, 1,000 of 2,048 4.1 and 6.5, 8,192 of 4,096
  // 9.4 and 12.3, 32,000 of 4,096 30.5 and 34.2, 2,048 of 16,384 13.9 and 17.8.  More tokens were measured with an earlier form of
  // that kernel only (one token of 8,192 channels 12.4 us): two, 8,192 of 4,096, 14.3 and 14.3, four, 32,000 of 4,096, 49 and 39.
  if (!a.x_scale && a.tokens == 1 && row <= kOwnBytes) {
    return eights<T>(a.x, a.x_ld, a.inputs) ? launch_own<T, true>(p, a.inputs, status, aligned, st)
                                            : launch_own<T, false>(p, a.inputs, status, aligned, st);
  }
  if (!a.x_scale) {
    const cortex_quant_i8_t q = {a.dtype, a.tokens, a.inputs, a.x, a.x_ld, rows, row, scales};
    const int rc = launch_quant<T>(q, status, (int)row, stream);
    if (rc != CORTEX_OK) return rc;
    p.x = rows;
    p.x_ld = row;
    p.x_scale = scales;
  } else if (a.inputs % kDepth || a.x_ld % 16 || a.x_ld > kMaxRow || !aligned16(a.x)) {
    pad_kernel<<<(unsigned)a.tokens, 256, 0, st>>>((const int8_t *)a.x, a.x_ld, a.inputs, rows, row, status);
    if (hipGetLastError() != hipSuccess) return CORTEX_E_HIP;
    p.x = rows;
    p.x_ld = row;
  }
  return launch_product<T>(p, status, aligned, st);
}

}  // namespace cortex

using namespace cortex;

extern "C" int cortex_quant_i8(const cortex_quant_i8_t *a, int32_t *status, void *stream) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (a->dtype != CORTEX_F32 && a->dtype != CORTEX_BF16) return CORTEX_E_INVAL;
  if (a->rows < 0 || a->rows >= kMaxRows || a->columns < 1 || a->columns > kMaxInputs) return CORTEX_E_INVAL;
  if (a->x_ld < a->columns || a->q_ld < a->columns) return CORTEX_E_INVAL;
  if (a->rows == 0) return CORTEX_OK;
  if (!a->x || !a->q || !a->scale) return CORTEX_E_INVAL;
  return a->dtype == CORTEX_BF16 ? launch_quant<bf16_t>(*a, status, a->columns, stream)
                                 : launch_quant<float>(*a, status, a->columns, stream);
}

extern "C" size_t cortex_linear_i8_workspace_bytes(int32_t tokens, int32_t outputs, int32_t inputs) {
  if (bad_linear_size(tokens, outputs, inputs)) return 0;
  return tokens ? linear_bytes(tokens, inputs) : 256;
}

extern "C" int cortex_linear_i8(const cortex_linear_i8_t *a, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (a->dtype != CORTEX_F32 && a->dtype != CORTEX_BF16) return CORTEX_E_INVAL;
  if (bad_linear_size(a->tokens, a->outputs, a->inputs) || a->tokens >= kMaxRows) return CORTEX_E_INVAL;
  if (a->x_ld < a->inputs || a->y_ld < a->outputs || a->w_ld < a->inputs || a->w_ld % 16 || a->w_ld > kMaxRow) return CORTEX_E_INVAL;
  if (a->tokens == 0) return CORTEX_OK;
  if (!a->x || !a->w || !a->w_scale || !a->y || !aligned16(a->w)) return CORTEX_E_INVAL;
  if (!ws || !aligned16(ws)) return CORTEX_E_INVAL;
  if (ws_bytes < linear_bytes(a->tokens, a->inputs)) return CORTEX_E_WORKSPACE;
  return a->dtype == CORTEX_BF16 ? launch_linear<bf16_t>(*a, status, ws, stream) : launch_linear<float>(*a, status, ws, stream);
}
