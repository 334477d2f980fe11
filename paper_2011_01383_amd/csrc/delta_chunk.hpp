// Prompts of the gated delta rule, as matrix products over chunks of 64 tokens.
//
// Within a chunk, with c_i = sum_{s <= i} dt_s A, the state S [V, K] that enters it and
//   L_ij = beta_i exp(c_i - c_j) (k_i . k_j)     j < i
//   P_ij = scale exp(c_i - c_j) (q_i . k_j)      j <= i
// the updates u_i = beta_i (v_i - exp(c_i) S k_i) - sum_{j < i} L_ij u_j are
//   U = T R,   T = (I + L)^-1,   R_i = beta_i (v_i - exp(c_i) S k_i)
// and the outputs and the next chunk's state
//   y_i = scale exp(c_i) S q_i + sum_{j <= i} P_ij u_j
//   S'  = exp(c_63) S + sum_j exp(c_63 - c_j) u_j k_j^T
// T and P depend on keys, queries and gates only: one launch makes them for all chunks
// at once (chunk_maps_kernel), and a second walks the chunks of a sequence, a workgroup 16 NT
// rows of one head's state (chunk_walk_kernel).
//
// Precision.  bf16 queries and keys enter the matrix units as they are, float32 ones and
// all that is computed on the way (T, P, R, U, the state) as three bf16 planes, eight bits
// each, which together are the value itself; of the products of two such, those
// below 2^-24 of the result are left out.  Sums are float32 and y is rounded once.
//
// Layouts.  A 16x16x32 product takes its operands as (index = lane & 15; 8 consecutive k
// from 8 (lane >> 4)) and leaves (column = lane & 15; rows 4 (lane >> 4) + 0..3).  Over tokens k
// = 8 q + 4 a + r stands for token 16 a + 4 q + r of each 32, and the rows of the state's
// tile a of each 32 entries are chosen as entries 8 q + 4 a + r: so what a lane
// ends with is what it hands on as eight bytes of a 16-byte operand.
#pragma once

#include "scan_head.hpp"

namespace cortex {

constexpr int kChunk = 64;
constexpr int kChunkWaves = 4;                   // 16 tokens each
constexpr int kChunkThreads = 64 * kChunkWaves;

// What the first launch leaves for a chunk and head.  Operand pieces of T and P: rows
// 16 w .. + 15, 32 tokens m = 0 .. w / 2; a lane's eight values in each of three planes.
constexpr int kMapPieces = 6;
// (For w < 2 there is no m = 1: its number names the wave's one piece.)
__device__ __forceinline__ constexpr int map_piece(int w, int m) { return w < 2 ? w : 2 * w - 2 + m; }
struct alignas(16) ChunkMap {
  u32x4v T[kMapPieces][3][64];
  u32x4v P[kMapPieces][3][64];
  float beta[kChunk];      // 0 past the sequence's end
  float grow[kChunk];      // exp(c_i)
  float weight[kChunk];    // exp(c_63 - c_i)
  float decay;             // exp(c_63)
  int first;               // first token that loses the whole head (not finite), or kChunk
  int pad[62];
};
static_assert(sizeof(ChunkMap) % 256 == 0, "maps start at 256 bytes");

template <typename T> constexpr int kKeyPlanes = sizeof(T) == 2 ? 1 : 3;

// a b summed into three accumulators by the size of their part, so that no product waits
// for the one before it; of three planes each only the six largest products.
struct Parts {
  f32x4 c[3];
  __device__ __forceinline__ Parts() {
#pragma unroll
    for (int s = 0; s < 3; ++s) c[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  template <int A, int B> __device__ __forceinline__ void add(const bf16x8v (&a)[A], const bf16x8v (&b)[B]) {
#pragma unroll
    for (int i = 0; i < A; ++i)
#pragma unroll
      for (int s = 2; s >= 0; --s)
        if (s - i >= 0 && s - i < B) c[s] = mfma_bf16x32(a[i], b[s - i], c[s]);
  }
  __device__ __forceinline__ f32x4 sum() const { return c[0] + (c[1] + c[2]); }
};

// Eight values as three planes.
__device__ __forceinline__ void planes8(float (&v)[8], bf16x8v (&p)[3]) {
  unsigned int b[4];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    plane(v, b);
    p[i] = pack8(b);
  }
}

// Eight elements of a key or query row as they are in memory, and their planes.
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4v v;
  template <bool WIDE> __device__ __forceinline__ void load(const bf16_t *p) { v = load8<WIDE>(p); }
  __device__ __forceinline__ void planes(bf16x8v (&f)[1]) const { f[0] = __builtin_bit_cast(bf16x8v, v); }
};
template <> struct Eight<float> {
  f32x4 lo, hi;
  template <bool WIDE> __device__ __forceinline__ void load(const float *p) {
    if constexpr (WIDE) {
      lo = *(const f32x4 *)p;
      hi = *(const f32x4 *)(p + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = p[i];
        hi[i] = p[4 + i];
      }
    }
  }
  __device__ __forceinline__ void planes(bf16x8v (&f)[3]) const {
    float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    planes8(v, f);
  }
};

// Inclusive sums over a wave, the sums' roundings in `low`.
__device__ __forceinline__ float exact_lane_sums(float v, float &low) {
  low = 0.0f;
  add_exactly(v, low, shifted<0x111>(v, 0.0f), shifted<0x111>(low, 0.0f));
  add_exactly(v, low, shifted<0x112>(v, 0.0f), shifted<0x112>(low, 0.0f));
  add_exactly(v, low, shifted<0x114>(v, 0.0f), shifted<0x114>(low, 0.0f));
  add_exactly(v, low, shifted<0x118>(v, 0.0f), shifted<0x118>(low, 0.0f));
  add_exactly(v, low, shifted<0x142, 0xa>(v, 0.0f), shifted<0x142, 0xa>(low, 0.0f));
  add_exactly(v, low, shifted<0x143, 0xc>(v, 0.0f), shifted<0x143, 0xc>(low, 0.0f));
  return v;
}

__device__ __forceinline__ bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }

// 16x16 blocks of float32 matrices in LDS: rows of 68 floats, so that rows lie 16
// bytes apart over the banks.
constexpr int kMatrixRow = kChunk + 4;
__device__ __forceinline__ f32x4 block_left(const float *m, int rb, int cb, int l16, int q) {
  return *(const f32x4 *)&m[(rb * 16 + l16) * kMatrixRow + cb * 16 + q * 4];
}
__device__ __forceinline__ f32x4 block_right(const float *m, int rb, int cb, int l16, int q) {
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = m[(rb * 16 + q * 4 + i) * kMatrixRow + cb * 16 + l16];
  return r;
}
// c + a b over 16: k = 4 q + step on both sides.  The result is a right operand as it stands.
__device__ __forceinline__ f32x4 mul_block(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// T and P of a chunk and head.  A wave has 16 rows of both; the products k . k and
// q . k are computed with the earlier token as the result's row, so a lane ends with four
// earlier tokens of its own row, which is how P is handed on.  T's blocks of 16 on the
// diagonal are inverted by substitution, a lane a column, then joined in two
// rounds: the corner below two inverses T1, T2 is - T2 L21 T1 (float32 matrix units).
template <typename T, int K, bool WIDE>
__global__ void __launch_bounds__(kChunkThreads, 2) chunk_maps_kernel(cortex_delta_t a, int32_t *status, ChunkMap *maps, int64_t units) {
  constexpr int KP = kKeyPlanes<T>, M = K / 32;
  __shared__ struct {
    alignas(16) float L[kChunk * kMatrixRow];
    alignas(16) float inverse[kChunk * kMatrixRow];
    alignas(16) float cum[kChunk], low[kChunk], beta[kChunk];
    int first;
  } lds;
  const int failed = entry_status(status);
  const int64_t unit = unit_of_block(units);
  if (unit >= units) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, w = tid >> 6, q = lane >> 4, l16 = lane & 15;
  const int slot = (int)(unit / a.heads), head = (int)(unit % a.heads), g = head / (a.heads / a.key_heads);
  if (head == 0) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, slot, status);
  const Chunk ch = find_chunk(a.seq_offsets, a.num_seqs, a.num_tokens, kChunk, slot);
  if (ch.seq < 0 || ch.begin == ch.end) return;
  if (tid == 0) lds.first = kChunk;
  if (__syncthreads_or(failed != 0)) return;
  ChunkMap &map = maps[(int64_t)slot * a.heads + head];
  const int last = ch.end - 1 - ch.begin;

  const T *ks = (const T *)a.k + (int64_t)ch.begin * a.k_ld + g * K + q * 8;
  const T *qs = (const T *)a.q + (int64_t)ch.begin * a.q_ld + g * K + q * 8;
  const int64_t own = min(w * 16 + l16, last);
  bf16x8v kf[M][KP], qf[M][KP];
  {
    Eight<T> kr[M], qr[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      kr[m].template load<WIDE>(ks + own * a.k_ld + m * 32);
      qr[m].template load<WIDE>(qs + own * a.q_ld + m * 32);
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      kr[m].planes(kf[m]);
      qr[m].planes(qf[m]);
    }
  }
  if (w == 0) {
    const int64_t t = ch.begin + min(lane, last);
    const bool live = lane <= last;
    float e = 0.0f;
    if (a.A) {
      const float raw = to_float<T>(((const T *)a.dt)[t * a.dt_ld + head]) + (a.dt_bias ? a.dt_bias[head] : 0.0f);
      e = (a.softplus ? softplus(raw) : raw) * decay_rate(a.A[head]);
    }
    const float b = to_float<T>(((const T *)a.b)[t * a.b_ld + head]);
    float beta = a.sigmoid ? sigmoid(b) : b;
    // An exponent is held to -256, which leaves nothing of the state, so that no sum is infinite.
    float held = e < -256.0f ? -256.0f : e;
    if (!live) beta = held = 0.0f;
    if (!finite(beta) || !finite(held)) {
      atomicMin(&lds.first, lane);
      beta = held = 0.0f;
    }
    float low, after_low;
    const float up = exact_lane_sums(held, low);
    const float down = exact_lane_sums(__shfl_xor(held, 63), after_low);      // from token 63 - lane on
    const float after = __shfl_up(down, 1);
    lds.cum[lane] = up;
    lds.low[lane] = low;
    lds.beta[lane] = beta;
    map.beta[lane] = beta;
    map.grow[lane] = fast_exp2(up);
    map.weight[63 - lane] = fast_exp2(lane == 0 ? 0.0f : after);
    if (lane == 63) map.decay = fast_exp2(down);
  }
  // a key that is not finite
  {
    bool odd = false;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const u32x4v bits = __builtin_bit_cast(u32x4v, kf[m][0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= (((bits[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0;
    }
    if (odd && w * 16 + l16 <= last) atomicMin(&lds.first, w * 16 + l16);
  }
  __syncthreads();
  const int i = w * 16 + l16;
  const float ci = lds.cum[i], li = lds.low[i], bi = lds.beta[i];
  float pv[2][4];
#pragma unroll
  for (int c = 0; c < kChunkWaves; ++c) {
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c <= w) {
      Parts kp, qp;
      const int64_t row = min(c * 16 + l16, last);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        Eight<T> raw;
        bf16x8v f[KP];
        raw.template load<WIDE>(ks + row * a.k_ld + m * 32);
        raw.planes(f);
        kp.add(f, kf[m]);
        qp.add(f, qf[m]);
      }
      const f32x4 kk = kp.sum(), qk = qp.sum();
      const int j0 = c * 16 + q * 4;
      const f32x4 cj = *(const f32x4 *)&lds.cum[j0], lj = *(const f32x4 *)&lds.low[j0];
      f32x4 l;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma clang fp reassociate(off)
        const float e = fast_exp2((ci - cj[r]) + (li - lj[r]));
        l[r] = j0 + r < i ? bi * e * kk[r] : 0.0f;
        v[r] = j0 + r <= i ? a.scale * e * qk[r] : 0.0f;
        if (!finite(l[r])) {
          atomicMin(&lds.first, i);
          l[r] = 0.0f;
        }
      }
      *(f32x4 *)&lds.L[i * kMatrixRow + j0] = l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) pv[c % 2][r] = v[r];
    if (c % 2 == 1 && c / 2 <= w / 2) {
      float e[8] = {pv[0][0], pv[0][1], pv[0][2], pv[0][3], pv[1][0], pv[1][1], pv[1][2], pv[1][3]};
      bf16x8v p[3];
      planes8(e, p);
#pragma unroll
      for (int n = 0; n < 3; ++n) map.P[map_piece(w, c / 2)][n][lane] = __builtin_bit_cast(u32x4v, p[n]);
    }
  }
  // The wave's own block on the diagonal: its rows were written by the wave itself.
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  {
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = r == l16 ? 1.0f : 0.0f;
#pragma unroll
      for (int s = 0; s < r; ++s) x[r] = __builtin_fmaf(-lds.L[(w * 16 + r) * kMatrixRow + w * 16 + s], x[s], x[r]);
      if (r / 4 == q) lds.inverse[(w * 16 + r) * kMatrixRow + w * 16 + l16] = x[r];
    }
  }
  __syncthreads();
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  auto put_block = [&](int rb, int cb, f32x4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) lds.inverse[(rb * 16 + q * 4 + r) * kMatrixRow + cb * 16 + l16] = -v[r];
  };
  if (w < 2) {
    const int b = 2 * w;
    const f32x4 x = mul_block(block_left(lds.L, b + 1, b, l16, q), block_right(lds.inverse, b, b, l16, q), zero);
    put_block(b + 1, b, mul_block(block_left(lds.inverse, b + 1, b + 1, l16, q), x, zero));
  }
  __syncthreads();
  {
    const int rb = 2 + w / 2, cb = w % 2;
    auto corner = [&](int s) {
      f32x4 y = zero;
      for (int c = cb; c < 2; ++c) y = mul_block(block_left(lds.L, s, c, l16, q), block_right(lds.inverse, c, cb, l16, q), y);
      return y;
    };
    f32x4 y = mul_block(block_left(lds.inverse, rb, 2, l16, q), corner(2), zero);
    if (rb == 3) y = mul_block(block_left(lds.inverse, 3, 3, l16, q), corner(3), y);
    put_block(rb, cb, y);
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    if (m > w / 2) break;
    float e[8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f32x4 v = zero;
      if (2 * m + s <= w) v = *(const f32x4 *)&lds.inverse[i * kMatrixRow + m * 32 + s * 16 + q * 4];
#pragma unroll
      for (int r = 0; r < 4; ++r) e[4 * s + r] = v[r];
    }
    bf16x8v p[3];
    planes8(e, p);
#pragma unroll
    for (int n = 0; n < 3; ++n) map.T[map_piece(w, m)][n][lane] = __builtin_bit_cast(u32x4v, p[n]);
  }
  if (tid == 0) map.first = lds.first;
}

// Products of planes, the largest part last: which plane of a and of b.
template <int A, int B> struct PlanePairs {
  static constexpr int kCount = A == 1 ? B : 6;
  static __device__ __forceinline__ constexpr int left(int i) { return A == 1 ? 0 : i == 0 || i == 3 ? 0 : i == 1 ? 1 : i == 2 ? 2 : i == 4 ? 1 : 0; }
  static __device__ __forceinline__ constexpr int right(int i) { return A == 1 ? B - 1 - i : i == 0 ? 2 : i == 1 ? 1 : i == 2 ? 0 : i == 3 ? 1 : 0; }
};

// The first of the tokens 16 tile + 4 q + r whose value is not finite; those values become 0: their
// products with the zeros above the diagonal would carry them to earlier tokens.
__device__ __forceinline__ void drop_odd(f32x4 (&v)[4], int q, int &first) {
#pragma clang fp reassociate(off)
  float none = 0.0f;
#pragma unroll
  for (int t = 0; t < 4; ++t) none += (v[t][0] * 0.0f + v[t][1] * 0.0f) + (v[t][2] * 0.0f + v[t][3] * 0.0f);
  if (!__any(none != 0.0f)) return;
#pragma unroll
  for (int t = 3; t >= 0; --t)
#pragma unroll
    for (int r = 3; r >= 0; --r)
      if (!finite(v[t][r])) {
        first = min(first, t * 16 + q * 4 + r);
        v[t][r] = 0.0f;
      }
  first = min(first, __shfl_xor(first, 16));
  first = min(first, __shfl_xor(first, 32));
}

template <typename T, int K> struct ChunkLds {
  static constexpr int KP = kKeyPlanes<T>;
  typedef Rows<K> K_;
  alignas(16) unsigned short keys[KP][kChunk * K_::kStride];
  alignas(16) unsigned short queries[KP][kChunk * K_::kStride];
  alignas(16) float beta[kChunk], grow[kChunk], weight[kChunk];
};

// A wave has 16 NT columns of the state (value channels) for all tokens and keys of its head, so
// what one product leaves is the next one's operand in the same lane and nothing goes
// between waves; a workgroup's waves share the keys and queries in LDS.
template <typename T, int K, int NT, bool WIDE>
__global__ void __launch_bounds__(kChunkThreads) chunk_walk_kernel(cortex_delta_t a, int32_t *status, const ChunkMap *maps, int64_t units) {
  typedef ChunkLds<T, K> Lds;
  constexpr int KP = Lds::KP, M = K / 32;
  constexpr int kItems = kChunk * (K / 8) / kChunkThreads;     // eights of keys that a thread brings in
  __shared__ Lds lds;
  const int failed = entry_status(status);
  const int64_t unit = unit_of_block(units);
  if (unit >= units) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, w = tid >> 6, q = lane >> 4, l16 = lane & 15;
  const int V = a.value_dim, wide = 16 * NT * kChunkWaves, slices = (V + wide - 1) / wide, per = a.heads * slices;
  const int seq = (int)(unit / per), rest = (int)(unit % per), head = rest / slices;
  const int v0 = rest % slices * wide + w * 16 * NT;
  const bool works = v0 < V;
  const int g = head / (a.heads / a.key_heads);
  const int begin = a.seq_offsets[seq], end = a.seq_offsets[seq + 1];
  if (begin < 0 || end < begin || end > a.num_tokens) return;
  int pool = -1;
  if (a.state_in || a.state_out) {
    pool = state_row(a.state_index, seq, a.state_rows, status);
    if (pool < -1) return;
  }
  if (__syncthreads_or(failed != 0)) return;
  // columns NT l16 .. + NT - 1; of the state's tile 2 m + s the lane has entries 32 m + 8 q + 4 s .. + 3
  const int col = works ? v0 + l16 * NT : 0;
  const int64_t state_at = (((int64_t)pool * a.heads + head) * V + col) * K + q * 8;
  f32x4 S[NT][2 * M];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int s = 0; s < 2 * M; ++s)
      S[n][s] = a.state_in && pool >= 0 && works ? *(const f32x4 *)(a.state_in + state_at + n * K + s / 2 * 32 + s % 2 * 4)
                                                 : f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const ChunkMap *map = maps + ((int64_t)(begin / kChunk) + seq) * a.heads + head;
  const T *ks = (const T *)a.k + g * K, *qs = (const T *)a.q + g * K;
  const T *vs = (const T *)a.v + (int64_t)head * V + col;
  T *ys = (T *)a.y + (int64_t)head * V + col;
  Eight<T> kr[kItems], qr[kItems];
  // Rows past the sequence's end repeat its last.
  auto load_rows = [&](int64_t t0) {
    const int last = (int)min((int64_t)kChunk, end - t0) - 1;
    const T *k0 = ks + t0 * a.k_ld, *q0 = qs + t0 * a.q_ld;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kChunkThreads + tid;
      const uint32_t row = min(id / (K / 8), last), o = id % (K / 8) * 8;
      kr[i].template load<WIDE>(k0 + (row * (uint32_t)a.k_ld + o));
      qr[i].template load<WIDE>(q0 + (row * (uint32_t)a.q_ld + o));
    }
  };
  if (begin < end) load_rows(begin);
#pragma unroll 1
  for (int64_t t0 = begin; t0 < end; t0 += kChunk, map += a.heads) {
    const int last = (int)min((int64_t)kChunk, end - t0) - 1;
    __syncthreads();                             // the last chunk's rows are read
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kChunkThreads + tid, at = Lds::K_::at(id / (K / 8), id % (K / 8) * 8);
      bf16x8v kf[KP], qf[KP];
      kr[i].planes(kf);
      qr[i].planes(qf);
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        *(u32x4v *)&lds.keys[p][at] = __builtin_bit_cast(u32x4v, kf[p]);
        *(u32x4v *)&lds.queries[p][at] = __builtin_bit_cast(u32x4v, qf[p]);
      }
    }
    if (tid < kChunk) {
      lds.beta[tid] = map->beta[tid];
      lds.grow[tid] = map->grow[tid];
      lds.weight[tid] = map->weight[tid];
    }
    u32x4v tr[kMapPieces][3];
#pragma unroll
    for (int i = 0; i < kMapPieces; ++i)
#pragma unroll
      for (int p = 0; p < 3; ++p) tr[i][p] = map->T[i][p][lane];
    T v[4][4][NT];
    const T *vt = vs + t0 * a.v_ld;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) v[t][r][n] = vt[(uint32_t)min(t * 16 + q * 4 + r, last) * (uint32_t)a.v_ld + n];
    const float decay = map->decay;
    int first[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) first[n] = map->first;
    load_rows(t0 + kChunk < end ? t0 + kChunk : t0);
    __syncthreads();                             // keys, queries and gates are there
    if (!works) continue;
    f32x4 kS[NT][4], y[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < 4; ++t) kS[n][t] = y[n][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf16x8v sp[NT][3], kf[4][KP], qf[4][KP];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float e[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          e[r] = S[n][2 * m][r];
          e[4 + r] = S[n][2 * m + 1][r];
        }
        planes8(e, sp[n]);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int p = 0; p < KP; ++p) {
          const int at = Lds::K_::at(t * 16 + l16, m * 32 + q * 8);
          kf[t][p] = lds8(&lds.keys[p][at]);
          qf[t][p] = lds8(&lds.queries[p][at]);
        }
      typedef PlanePairs<KP, 3> Pairs;
#pragma unroll
      for (int i = 0; i < Pairs::kCount; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            kS[n][t] = mfma_bf16x32(kf[t][Pairs::left(i)], sp[n][Pairs::right(i)], kS[n][t]);
            y[n][t] = mfma_bf16x32(qf[t][Pairs::left(i)], sp[n][Pairs::right(i)], y[n][t]);
          }
    }
    typedef PlanePairs<3, 3> Pairs;
    bf16x8v rp[NT][2][3], up[NT][2][3], wp[NT][2][3];
    auto to_planes = [](const f32x4 &lo, const f32x4 &hi, bf16x8v (&p)[3]) {
      float e[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      planes8(e, p);
    };
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4 beta = *(const f32x4 *)&lds.beta[t * 16 + q * 4], grow = *(const f32x4 *)&lds.grow[t * 16 + q * 4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = beta[r] * (to_float<T>(v[t][r][n]) - grow[r] * kS[n][t][r]);
          kS[n][t][r] = t * 16 + q * 4 + r <= last ? x : 0.0f;
          y[n][t][r] *= a.scale * grow[r];
        }
      }
      drop_odd(kS[n], q, first[n]);
#pragma unroll
      for (int m = 0; m < 2; ++m) to_planes(kS[n][2 * m], kS[n][2 * m + 1], rp[n][m]);
    }
    f32x4 u[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < 4; ++t) u[n][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < Pairs::kCount; ++i)
#pragma unroll
        for (int t = 2 * m; t < 4; ++t)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            u[n][t] = mfma_bf16x32(__builtin_bit_cast(bf16x8v, tr[map_piece(t, m)][Pairs::left(i)]), rp[n][m][Pairs::right(i)], u[n][t]);
#pragma unroll
    for (int i = 0; i < kMapPieces; ++i)
#pragma unroll
      for (int p = 0; p < 3; ++p) tr[i][p] = map->P[i][p][lane];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      drop_odd(u[n], q, first[n]);
      f32x4 weighted[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) weighted[t] = u[n][t] * *(const f32x4 *)&lds.weight[t * 16 + q * 4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        to_planes(u[n][2 * m], u[n][2 * m + 1], up[n][m]);
        to_planes(weighted[2 * m], weighted[2 * m + 1], wp[n][m]);
      }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf16x8v kt[2][2][KP];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int n = 0; n < NT; ++n) S[n][2 * m + s] *= decay;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = Lds::K_::at(h * 32 + q * 4 + l16 / 4, m * 32 + l16 % 4 * 8 + s * 4);
          const int to = Lds::K_::at(h * 32 + 16 + q * 4 + l16 / 4, m * 32 + l16 % 4 * 8 + s * 4);
#pragma unroll
          for (int p = 0; p < KP; ++p) kt[s][h][p] = join8(lds_columns(&lds.keys[p][at]), lds_columns(&lds.keys[p][to]));
        }
      }
      typedef PlanePairs<KP, 3> KeyPairs;
#pragma unroll
      for (int i = 0; i < KeyPairs::kCount; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              S[n][2 * m + s] = mfma_bf16x32(kt[s][h][KeyPairs::left(i)], wp[n][h][KeyPairs::right(i)], S[n][2 * m + s]);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < Pairs::kCount; ++i)
#pragma unroll
        for (int t = 2 * m; t < 4; ++t)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            y[n][t] = mfma_bf16x32(__builtin_bit_cast(bf16x8v, tr[map_piece(t, m)][Pairs::left(i)]), up[n][m][Pairs::right(i)], y[n][t]);
    T *yt = ys + t0 * a.y_ld;
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (__any(first[n] < kChunk)) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (t * 16 + q * 4 + r >= first[n]) y[n][t][r] = __builtin_nanf("");
        if (first[n] < kChunk)
#pragma unroll
          for (int s = 0; s < 2 * M; ++s) S[n][s] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
      }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (t * 16 + q * 4 + r <= last)
#pragma unroll
          for (int n = 0; n < NT; ++n) yt[(uint32_t)(t * 16 + q * 4 + r) * (uint32_t)a.y_ld + n] = from_float<T>(y[n][t][r]);
  }
  if (a.state_out && pool >= 0 && works)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int s = 0; s < 2 * M; ++s) *(f32x4 *)(a.state_out + state_at + n * K + s / 2 * 32 + s % 2 * 4) = S[n][s];
}

// Four values of one column as the lane's half of an operand, three planes.
__device__ __forceinline__ void put_planes4(u32x4v *to, int plane_stride, int lane, int half, f32x4 x) {
  float v[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    unsigned int b[2];
    plane(v, b);
    *(u32x2v *)((char *)(to + n * plane_stride + lane) + 8 * half) = u32x2v{b[0], b[1]};
  }
}

template <typename T, int K> struct ChainLds {
  static constexpr int KP = kKeyPlanes<T>, M = K / 32;
  typedef Rows<K> K_;
  alignas(16) u32x4v S[3][M][64];
  alignas(16) u32x4v R[3][2][64];
  alignas(16) u32x4v W[3][2][64];                // exp(c_63 - c_j) u_j
  alignas(16) f32x4 U[4][64];
  alignas(16) unsigned short keys[KP][kChunk * K_::kStride];
  int first[2][16];
};

// The same for few columns: eight waves share 16 of them, so that the chain from one state to
// the next is short.  Four waves of 16 tokens each form it: keys by state, R; U; the
// next state, an LDS exchange and a barrier between; four more form the outputs beside them.
template <typename T, int K, bool WIDE>
__global__ void __launch_bounds__(2 * kChunkThreads) chunk_chain_kernel(cortex_delta_t a, int32_t *status, const ChunkMap *maps, int64_t units) {
  typedef ChainLds<T, K> Lds;
  constexpr int KP = Lds::KP, M = Lds::M;
  constexpr int ST = K == 128 ? 2 : 1;           // tiles of 16 state entries of a wave
  __shared__ Lds lds;
  const int failed = entry_status(status);
  const int64_t unit = unit_of_block(units);
  if (unit >= units) return;
  const int tid = (int)threadIdx.x, lane = tid & 63, q = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), w = wave & 3;
  const int V = a.value_dim, slices = V / 16, per = a.heads * slices;
  const int seq = (int)(unit / per), rest = (int)(unit % per), head = rest / slices, v0 = rest % slices * 16;
  const int g = head / (a.heads / a.key_heads);
  const int begin = a.seq_offsets[seq], end = a.seq_offsets[seq + 1];
  if (begin < 0 || end < begin || end > a.num_tokens) return;
  int pool = -1;
  if (a.state_in || a.state_out) {
    pool = state_row(a.state_index, seq, a.state_rows, status);
    if (pool < -1) return;
  }
  if (__syncthreads_or(failed != 0)) return;
  const ChunkMap *map = maps + ((int64_t)(begin / kChunk) + seq) * a.heads + head;
  // What a chunk needs is loaded as soon as the last chunk's is used up, without a condition, so
  // that nothing waits for it: the last chunk repeats its own.  Rows past the sequence's end
  // repeat its last.  Places in a chunk are 32 bits (the host admits no longer rows).
  u32x4v piece[2][3];
  auto load_pieces = [&](const u32x4v (&of)[kMapPieces][3][64]) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int p = 0; p < 3; ++p) piece[m][p] = of[map_piece(w, m)][p][lane];
  };
  Eight<T> raw[M];
  uint32_t own = 0;
  auto load_own = [&](const T *rows) {
#pragma unroll
    for (int m = 0; m < M; ++m) raw[m].template load<WIDE>(rows + own + m * 32);
  };
  int b = 0;
  if (wave >= kChunkWaves) {
    const T *qs = (const T *)a.q + g * K + q * 8;
    T *ys = (T *)a.y + (int64_t)head * V + v0 + l16;
    uint32_t y_at[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) y_at[r] = (uint32_t)(w * 16 + q * 4 + r) * (uint32_t)a.y_ld;
    f32x4 grow = {0.0f, 0.0f, 0.0f, 0.0f};
    if (begin < end) {
      own = (uint32_t)min(w * 16 + l16, min(kChunk, end - begin) - 1) * (uint32_t)a.q_ld;
      load_own(qs + (int64_t)begin * a.q_ld);
      load_pieces(map->P);
      grow = *(const f32x4 *)&map->grow[w * 16 + q * 4];
    }
#pragma unroll 1
    for (int64_t t0 = begin; t0 < end; t0 += kChunk, b ^= 1) {
      const int last = (int)min((int64_t)kChunk, end - t0) - 1;
      const bool more = t0 + kChunk < end;
      const int64_t next = more ? t0 + kChunk : t0;
      if (more) map += a.heads;
      __syncthreads();                           // the state is there
      Parts qp;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        bf16x8v f[KP], s[3];
        raw[m].planes(f);
#pragma unroll
        for (int p = 0; p < 3; ++p) s[p] = __builtin_bit_cast(bf16x8v, lds.S[p][m][lane]);
        qp.add(f, s);
      }
      f32x4 y = qp.sum() * (grow * a.scale);
      if (end - next < kChunk) own = (uint32_t)min(w * 16 + l16, (int)(end - next) - 1) * (uint32_t)a.q_ld;
      load_own(qs + next * a.q_ld);
      grow = *(const f32x4 *)&map->grow[w * 16 + q * 4];
      __syncthreads();                           // R is there
      __syncthreads();                           // U is there
      Parts yp;
#pragma unroll
      for (int m = 0; m < 2; ++m)
        if (m <= w / 2) {
          const f32x4 lo = lds.U[2 * m][lane], hi = lds.U[2 * m + 1][lane];
          float e[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          bf16x8v p3[3], s[3];
          planes8(e, s);
#pragma unroll
          for (int p = 0; p < 3; ++p) p3[p] = __builtin_bit_cast(bf16x8v, piece[m][p]);
          yp.add(p3, s);
        }
      y += yp.sum();
      load_pieces(map->P);
      const int from = lds.first[b][l16];
      T *yt = ys + t0 * a.y_ld;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = w * 16 + q * 4 + r;
        if (i <= last) yt[y_at[r]] = from_float<T>(i < from ? y[r] : __builtin_nanf(""));
      }
    }
    return;
  }
  __builtin_amdgcn_s_setprio(2);                 // the outputs have time until the next state
  // the wave's part of the state: 32 entries m, its halves of four in eight from `half` on
  const int sm = K == 128 ? w : K == 64 ? w / 2 : 0, half = K == 128 ? 0 : K == 64 ? w % 2 : w;
  const bool holds = K > 32 || w < 2;
  const int64_t state_at = (((int64_t)pool * a.heads + head) * V + v0 + l16) * K + sm * 32 + q * 8 + half * 4;
  f32x4 S[ST];
  auto put_state = [&]() {
    if (!holds) return;
#pragma unroll
    for (int s = 0; s < ST; ++s) put_planes4(&lds.S[0][sm][0], M * 64, lane, half + s, S[s]);
  };
#pragma unroll
  for (int s = 0; s < ST; ++s)
    S[s] = a.state_in && pool >= 0 && holds ? *(const f32x4 *)(a.state_in + state_at + s * 4) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  put_state();
  const T *ks = (const T *)a.k + g * K + q * 8, *vs = (const T *)a.v + (int64_t)head * V + v0 + l16;
  T v[4];
  uint32_t v_at[4] = {};
  struct Gates {
    f32x4 beta, grow, weight;
    float decay;
    int first;
  } gates, coming = {};
  auto place_rows = [&](int last) {
    own = (uint32_t)min(w * 16 + l16, last) * (uint32_t)a.k_ld;
#pragma unroll
    for (int r = 0; r < 4; ++r) v_at[r] = (uint32_t)min(w * 16 + q * 4 + r, last) * (uint32_t)a.v_ld;
  };
  auto load_rows = [&](int64_t t0) {
    load_own(ks + t0 * a.k_ld);
    const T *vt = vs + t0 * a.v_ld;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = vt[v_at[r]];
  };
  auto load_gates = [&]() {
    coming.beta = *(const f32x4 *)&map->beta[w * 16 + q * 4];
    coming.grow = *(const f32x4 *)&map->grow[w * 16 + q * 4];
    coming.weight = *(const f32x4 *)&map->weight[w * 16 + q * 4];
    coming.decay = map->decay;
    coming.first = map->first;
  };
  // Values of the lane's tokens that are not finite become 0: their products with the zeros above
  // the diagonal would carry them to earlier tokens.  The first is noted.
  auto drop = [&](f32x4 &x) {
#pragma clang fp reassociate(off)
    const float none = (x[0] * 0.0f + x[1] * 0.0f) + (x[2] * 0.0f + x[3] * 0.0f);
    if (none == 0.0f) return;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!finite(x[r])) {
        atomicMin(&lds.first[b][l16], w * 16 + q * 4 + r);
        x[r] = 0.0f;
      }
  };
  if (begin < end) {
    load_gates();
    place_rows(min(kChunk, end - begin) - 1);
    load_rows(begin);
    load_pieces(map->T);
  }
#pragma unroll 1
  for (int64_t t0 = begin; t0 < end; t0 += kChunk, b ^= 1) {
    const int last = (int)min((int64_t)kChunk, end - t0) - 1;
    const bool more = t0 + kChunk < end;
    const int64_t next = more ? t0 + kChunk : t0;
    if (more) map += a.heads;
    gates = coming;
    load_gates();
    if (tid < 16) lds.first[b][tid] = gates.first;
    __syncthreads();                             // the state is there; the last chunk's keys are read
    bf16x8v kf[M][KP];
#pragma unroll
    for (int m = 0; m < M; ++m) raw[m].planes(kf[m]);
    Parts kp;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf16x8v s[3];
#pragma unroll
      for (int p = 0; p < 3; ++p) s[p] = __builtin_bit_cast(bf16x8v, lds.S[p][m][lane]);
      kp.add(kf[m], s);
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int p = 0; p < KP; ++p)
        *(u32x4v *)&lds.keys[p][Lds::K_::at(w * 16 + l16, m * 32 + q * 8)] = __builtin_bit_cast(u32x4v, kf[m][p]);
    f32x4 x = kp.sum();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[r] = gates.beta[r] * (to_float<T>(v[r]) - gates.grow[r] * x[r]);
      if (w * 16 + q * 4 + r > last) x[r] = 0.0f;
    }
    drop(x);
    put_planes4(&lds.R[0][w / 2][0], 2 * 64, lane, w % 2, x);
    if (end - next < kChunk) place_rows((int)(end - next) - 1);
    load_rows(next);
    __syncthreads();                             // R and the keys are there
    Parts up;
#pragma unroll
    for (int m = 0; m < 2; ++m)
      if (m <= w / 2) {
        bf16x8v t[3], s[3];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          t[p] = __builtin_bit_cast(bf16x8v, piece[m][p]);
          s[p] = __builtin_bit_cast(bf16x8v, lds.R[p][m][lane]);
        }
        up.add(t, s);
      }
    bf16x8v kt[ST][2][KP];
    if (holds)
#pragma unroll
      for (int s = 0; s < ST; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const int at = Lds::K_::at(m * 32 + q * 4 + l16 / 4, sm * 32 + l16 % 4 * 8 + (half + s) * 4);
          const int to = Lds::K_::at(m * 32 + 16 + q * 4 + l16 / 4, sm * 32 + l16 % 4 * 8 + (half + s) * 4);
#pragma unroll
          for (int p = 0; p < KP; ++p) kt[s][m][p] = join8(lds_columns(&lds.keys[p][at]), lds_columns(&lds.keys[p][to]));
        }
    f32x4 u = up.sum();
    drop(u);
    put_planes4(&lds.W[0][w / 2][0], 2 * 64, lane, w % 2, u * gates.weight);
    lds.U[w][lane] = u;
    load_pieces(map->T);
    __syncthreads();                             // U is there
    if (holds) {
      const bool gone = lds.first[b][l16] < kChunk;
      Parts sp[ST];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        bf16x8v x3[3];
#pragma unroll
        for (int p = 0; p < 3; ++p) x3[p] = __builtin_bit_cast(bf16x8v, lds.W[p][m][lane]);
#pragma unroll
        for (int s = 0; s < ST; ++s) sp[s].add(kt[s][m], x3);
      }
#pragma unroll
      for (int s = 0; s < ST; ++s) {
        S[s] = S[s] * gates.decay + sp[s].sum();
        if (gone) S[s] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
      }
    }
    put_state();
  }
  if (a.state_out && pool >= 0 && holds)
#pragma unroll
    for (int s = 0; s < ST; ++s) *(f32x4 *)(a.state_out + state_at + s * 4) = S[s];
}

}  // namespace cortex
