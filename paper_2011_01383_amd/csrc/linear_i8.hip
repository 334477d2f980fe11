// Rows to 8 bits, and the projection that multiplies them.
//
// Weights are the first operand of the matrix units and tokens the second, so a
// lane ends with four neighbouring channels of one token.
#include "sequence.hpp"

namespace cortex {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int32_t kMaxInputs = 131071;           // 128 * 128 of each stay below 2^31

// ---------------------------------------------------------------------------
// Rows to 8 bits
// ---------------------------------------------------------------------------
constexpr int kQuantThreads = 256;

// One value: x / scale rounded to a whole number.  A scale in the denormals may
// leave the quotient above 127.
__device__ __forceinline__ int quant_value(float x, float scale) {
  const float v = __builtin_rintf(x / scale);
  return (int)__builtin_fminf(__builtin_fmaxf(v, -127.0f), 127.0f);
}

// `filled`: columns of q that are written, zeros past the row's own.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kQuantThreads) quant_kernel(cortex_quant_i8_t a, int32_t *status, int filled) {
  constexpr int V = WIDE ? 8 : 1;
  __shared__ unsigned int most[kQuantThreads / 64];
  if (__syncthreads_or(entry_status(status) != 0)) return;
  const int tid = (int)threadIdx.x;
  const int64_t r = blockIdx.x;
  const T *x = (const T *)a.x + r * a.x_ld;
  int8_t *q = a.q + r * a.q_ld;
  // |x| as whole numbers keep their order; infinities and NaN are the largest
  unsigned int top = 0;
  for (int c = tid * V; c < a.columns; c += kQuantThreads * V) {
    float v[V];
    Pack<T, V>::load(x + c, v);
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __builtin_bit_cast(unsigned int, v[i]) & 0x7fffffffu);
  }
#pragma unroll
  for (int m = 32; m; m >>= 1) top = max(top, (unsigned int)__shfl_xor((int)top, m));
  if ((tid & 63) == 0) most[tid >> 6] = top;
  __syncthreads();
  top = max(max(most[0], most[1]), max(most[2], most[3]));
  const bool odd = top >= 0x7f800000u;
  const float scale = odd ? __builtin_nanf("") : __builtin_bit_cast(float, top) / 127.0f;
  const bool none = odd || scale == 0.0f;
  for (int c = tid * V; c < filled; c += kQuantThreads * V) {
    float v[V];
    int8_t to[V];
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = 0;
    if (c < a.columns) {
      Pack<T, V>::load(x + c, v);
#pragma unroll
      for (int i = 0; i < V; ++i) to[i] = none ? 0 : (int8_t)quant_value(v[i], scale);
    }
    if constexpr (WIDE) {
      typedef int8_t pack __attribute__((ext_vector_type(8)));
      *(pack *)(q + c) = pack{to[0], to[1], to[2], to[3], to[4], to[5], to[6], to[7]};
    } else {
      q[c] = to[0];
    }
  }
  if (tid == 0) a.scale[r] = scale;
}

template <typename T> int launch_quant(const cortex_quant_i8_t &a, int32_t *status, int filled, void *stream) {
  constexpr uintptr_t mask = sizeof(T) == 2 ? 15 : 31;
  const bool wide = a.columns % 8 == 0 && filled % 8 == 0 && a.x_ld % 8 == 0 && a.q_ld % 8 == 0 && ((uintptr_t)a.x & mask) == 0 &&
                    ((uintptr_t)a.q & 7) == 0;
  const hipStream_t st = (hipStream_t)stream;
  if (wide) quant_kernel<T, true><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a, status, filled);
  else quant_kernel<T, false><<<(unsigned)a.rows, kQuantThreads, 0, st>>>(a, status, filled);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
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
// What a product kernel takes: x in rows of whole 16-byte pieces, zeros past the
// inputs; `pieces` of them hold inputs.
struct Product {
  const int8_t *x, *w;
  int64_t x_ld, w_ld, y_ld;
  const float *x_scale, *w_scale, *bias;
  void *y;
  int32_t tokens, outputs, pieces;
};

template <typename T> __device__ __forceinline__ T finish(const Product &a, int acc, float xs, int n) {
#pragma clang fp contract(off)
  float v = (float)acc * xs * a.w_scale[n];
  if (a.bias) v += a.bias[n];
  return from_float<T>(v);
}

constexpr int kTile = 128, kDepth = 128;         // channels or tokens of a tile, bytes of the inputs at a time

// A row of 128 bytes in LDS, its 16-byte pieces exchanged so that the rows and pieces
// that the hardware serves together (rows 0-3 and 12-15 of sixteen with rows 4-11 of
// the next piece) lie in different banks.
__device__ __forceinline__ int piece_at(int row, int piece) { return row * kDepth + ((piece ^ ((row >> 1) & 7)) << 4); }

template <typename T>
__global__ void __launch_bounds__(256) product_kernel(Product a, const int32_t *status, bool aligned) {
  __shared__ __attribute__((aligned(16))) int8_t lds[2][2][kTile * kDepth];
  if (__syncthreads_or(entry_status(status) != 0)) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4, l16 = lane & 15;
  const int n0 = (int)blockIdx.x * kTile, t0 = (int)blockIdx.y * kTile;
  const int wn = wave % 2 * 64, wt = wave / 2 * 64;
  i32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  i32x4 wr[4], xr[4];
  auto fetch = [&](int p0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = i * 256 + tid, row = id / 8, p = p0 + id % 8;
      wr[i] = xr[i] = i32x4{0, 0, 0, 0};
      if (p < a.pieces) {
        wr[i] = *(const i32x4 *)(a.w + (int64_t)min(n0 + row, a.outputs - 1) * a.w_ld + (int64_t)p * 16);
        xr[i] = *(const i32x4 *)(a.x + (int64_t)min(t0 + row, a.tokens - 1) * a.x_ld + (int64_t)p * 16);
      }
    }
  };
  auto put = [&](int b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int id = i * 256 + tid;
      *(i32x4 *)&lds[b][0][piece_at(id / 8, id % 8)] = wr[i];
      *(i32x4 *)&lds[b][1][piece_at(id / 8, id % 8)] = xr[i];
    }
  };
  fetch(0);
  put(0);
  __syncthreads();
  int b = 0;
#pragma unroll 1
  for (int p0 = 0; p0 < a.pieces; p0 += 8, b ^= 1) {
    if (p0 + 8 < a.pieces) fetch(p0 + 8);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      i32x4 w[4], x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = *(const i32x4 *)&lds[b][0][piece_at(wn + i * 16 + l16, m * 4 + q)];
        x[i] = *(const i32x4 *)&lds[b][1][piece_at(wt + i * 16 + l16, m * 4 + q)];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
    }
    if (p0 + 8 < a.pieces) put(b ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int t = t0 + wt + j * 16 + l16;
    if (t >= a.tokens) continue;
    const float xs = a.x_scale[t];
    T *y = (T *)a.y + (int64_t)t * a.y_ld;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + wn + i * 16 + q * 4;
      if (aligned && n + 3 < a.outputs) {
        typedef T pack __attribute__((ext_vector_type(4)));
        pack v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = finish<T>(a, acc[i][j][r], xs, n + r);
        *(pack *)(y + n) = v;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < a.outputs) y[n + r] = finish<T>(a, acc[i][j][r], xs, n + r);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The call
// ---------------------------------------------------------------------------
// The workspace: tokens in 8 bits, in rows of a multiple of 16 bytes, and their scales.
static int64_t row_bytes(int32_t inputs) { return ((int64_t)inputs + 15) / 16 * 16; }
static size_t linear_bytes(int64_t tokens, int32_t inputs) {
  return align_up((size_t)(tokens * row_bytes(inputs)), 256) + align_up((size_t)tokens * 4, 256);
}

static bool bad_linear_size(int32_t tokens, int32_t outputs, int32_t inputs) {
  return tokens < 0 || outputs < 1 || inputs < 1 || inputs > kMaxInputs;
}

template <typename T> int launch_linear(const cortex_linear_i8_t &a, int32_t *status, void *ws, void *stream) {
  const hipStream_t st = (hipStream_t)stream;
  const int64_t row = row_bytes(a.inputs);
  Product p = {(const int8_t *)a.x, a.w, a.x_ld, a.w_ld, a.y_ld, a.x_scale, a.w_scale, a.bias, a.y, a.tokens, a.outputs, (int32_t)(row / 16)};
  int8_t *rows = (int8_t *)ws;
  float *scales = (float *)(rows + align_up((size_t)(a.tokens * row), 256));
  if (!a.x_scale) {
    const cortex_quant_i8_t q = {a.dtype, a.tokens, a.inputs, a.x, a.x_ld, rows, row, scales};
    const int rc = launch_quant<T>(q, status, (int)row, stream);
    if (rc != CORTEX_OK) return rc;
    p.x = rows;
    p.x_ld = row;
    p.x_scale = scales;
  } else if (a.inputs % 16 || a.x_ld % 16 || !aligned16(a.x)) {
    pad_kernel<<<(unsigned)a.tokens, 256, 0, st>>>((const int8_t *)a.x, a.x_ld, a.inputs, rows, row, status);
    if (hipGetLastError() != hipSuccess) return CORTEX_E_HIP;
    p.x = rows;
    p.x_ld = row;
  }
  const bool aligned = a.y_ld % 4 == 0 && ((uintptr_t)a.y & (4 * sizeof(T) - 1)) == 0;
  product_kernel<T><<<dim3((a.outputs + kTile - 1) / kTile, (a.tokens + kTile - 1) / kTile), 256, 0, st>>>(p, status, aligned);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

}  // namespace cortex

using namespace cortex;

extern "C" int cortex_quant_i8(const cortex_quant_i8_t *a, int32_t *status, void *stream) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (a->dtype != CORTEX_F32 && a->dtype != CORTEX_BF16) return CORTEX_E_INVAL;
  // a workgroup of 256 a row, and a grid has less than 2^32 threads
  if (a->rows < 0 || a->rows >= 1 << 24 || a->columns < 1 || a->columns > kMaxInputs) return CORTEX_E_INVAL;
  if (a->x_ld < a->columns || a->q_ld < a->columns) return CORTEX_E_INVAL;
  if (a->rows == 0) return CORTEX_OK;
  if (!a->x || !a->q || !a->scale) return CORTEX_E_INVAL;
  return a->dtype == CORTEX_BF16 ? launch_quant<bf16_t>(*a, status, a->columns, stream)
                                 : launch_quant<float>(*a, status, a->columns, stream);
}

extern "C" size_t cortex_linear_i8_workspace_bytes(int32_t tokens, int32_t outputs, int32_t inputs) {
  return bad_linear_size(tokens, outputs, inputs) ? 0 : linear_bytes(tokens, inputs) + 16;
}

extern "C" int cortex_linear_i8(const cortex_linear_i8_t *a, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (a->dtype != CORTEX_F32 && a->dtype != CORTEX_BF16) return CORTEX_E_INVAL;
  // tiles of tokens are counted in 16 bits
  if (bad_linear_size(a->tokens, a->outputs, a->inputs) || a->tokens > 65535 * kTile) return CORTEX_E_INVAL;
  if (a->x_ld < a->inputs || a->y_ld < a->outputs || a->w_ld < row_bytes(a->inputs) || a->w_ld % 16) return CORTEX_E_INVAL;
  if (a->tokens == 0) return CORTEX_OK;
  if (!a->x || !a->w || !a->w_scale || !a->y || !aligned16(a->w)) return CORTEX_E_INVAL;
  if (!ws || !aligned16(ws)) return CORTEX_E_INVAL;
  if (ws_bytes < linear_bytes(a->tokens, a->inputs)) return CORTEX_E_WORKSPACE;
  return a->dtype == CORTEX_BF16 ? launch_linear<bf16_t>(*a, status, ws, stream) : launch_linear<float>(*a, status, ws, stream);
}
