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
// at once (chunk_maps_kernel), and a second walks the chunks of a sequence: with a wave to 16
// rows of a head's state where there are many (chunk_walk_kernel), a workgroup where there are few
// (chunk_chain_kernel).
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
constexpr int kChainThreads = 2 * kChunkThreads + 64;

// What the first launch leaves for a chunk and head.  Operand pieces of T: rows
// 16 w .. + 15, 32 tokens m = 0 .. w / 2; a lane's eight values in each of three planes.
constexpr int kMapPieces = 6;
// (For w < 2 there is no m = 1: its number names the wave's one piece.)
__device__ __forceinline__ constexpr int map_piece(int w, int m) { return w < 2 ? w : 2 * w - 2 + m; }
// Tiles of P: rows 16 w .. + 15 by tokens 16 c .. + 15, c <= w; a lane has tokens 4 q .. + 3 of row lane & 15.
constexpr int kMapTiles = 10;
__device__ __forceinline__ constexpr int map_tile(int w, int c) { return w * (w + 1) / 2 + c; }
enum { kBeta, kGrow, kWeight, kRest, kGates };
struct alignas(16) ChunkMap {
  u32x4v T[kMapPieces][3][64];
  union {
    f32x4 P[kMapTiles][64];
    u32x4v pieces[kMapPieces][3][64];            // of P, as T's
  };
  // beta_i (0 past the sequence's end); exp(c_i); exp(c_63 - c_i); then exp(c_63) and the first token
  // that loses the whole head (not finite), or kChunk.
  float gates[kGates][kChunk];
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

// T, P and the gates of a chunk and head.  A wave has 16 rows; the products k . k and q . k are computed with
// the earlier token as the result's row, so a lane ends with four earlier tokens of its own row.
// T's blocks of 16 on the diagonal are inverted by substitution, a lane a column, then
// joined in two rounds: the corner below two inverses T1, T2 is - T2 L21 T1 (float32 matrix
// units).  A block of T takes the place of L's once that is used up.
//
// Chunks do not depend on each other, so there are as many workgroups as chunks and heads, and what bounds it is the
// latency of one: substitution, two rounds of blocks and four barriers, each with little work.  8,192 tokens of 32 heads of
// 128 (16 prompts) take 63 us and write some 170 MB, 32,768 tokens 180 (with nothing stored 134).  PIECES: P is left as planes,
// which every wave of the walk reads, else as float32 tiles, which are fewer bytes for the chain to copy.
template <typename T, int K, bool PIECES, bool WIDE>
__global__ void __launch_bounds__(kChunkThreads, 4) chunk_maps_kernel(cortex_delta_t a, int32_t *status, ChunkMap *maps, int64_t units) {
  constexpr int KP = kKeyPlanes<T>, M = K / 32;
  typedef Rows<K> K_;
  __shared__ struct {
    union {
      alignas(16) float L[kChunk * kMatrixRow];
      alignas(16) unsigned short keys[KP][kChunk * K_::kStride];
    };
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
  const int last = ch.end - 1 - ch.begin, i = w * 16 + l16;

  const T *ks = (const T *)a.k + (int64_t)ch.begin * a.k_ld + g * K + q * 8;
  const T *qs = (const T *)a.q + (int64_t)ch.begin * a.q_ld + g * K + q * 8;
  bf16x8v kf[M][KP], qf[M][KP];
  {
    Eight<T> raw[M], qr[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      raw[m].template load<WIDE>(ks + (int64_t)min(i, last) * a.k_ld + m * 32);
      qr[m].template load<WIDE>(qs + (int64_t)min(i, last) * a.q_ld + m * 32);
    }
    if (w == 0) {
      const int64_t t = ch.begin + min(lane, last);
      float e = 0.0f;
      if (a.A) {
        const float v = to_float<T>(((const T *)a.dt)[t * a.dt_ld + head]) + (a.dt_bias ? a.dt_bias[head] : 0.0f);
        e = (a.softplus ? softplus(v) : v) * decay_rate(a.A[head]);
      }
      const float b = to_float<T>(((const T *)a.b)[t * a.b_ld + head]);
      float beta = a.sigmoid ? sigmoid(b) : b;
      // An exponent is held to -256, which leaves nothing of the state, so that no sum is infinite.
      float held = e < -256.0f ? -256.0f : e;
      if (lane > last) beta = held = 0.0f;
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
      map.gates[kBeta][lane] = beta;
      map.gates[kGrow][lane] = fast_exp2(up);
      map.gates[kWeight][63 - lane] = fast_exp2(lane == 0 ? 0.0f : after);
      if (lane == 63) map.gates[kRest][0] = fast_exp2(down);
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      raw[m].planes(kf[m]);
      qr[m].planes(qf[m]);
    }
  }
  // a key that is not finite
  {
    bool odd = false;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const u32x4v bits = __builtin_bit_cast(u32x4v, kf[m][0]);
#pragma unroll
      for (int r = 0; r < 4; ++r) odd |= (((bits[r] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0;
    }
    if (odd && i <= last) atomicMin(&lds.first, i);
  }
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int p = 0; p < KP; ++p) *(u32x4v *)&lds.keys[p][K_::at(i, m * 32 + q * 8)] = __builtin_bit_cast(u32x4v, kf[m][p]);
  __syncthreads();
  f32x4 l[kChunkWaves], s[kChunkWaves];
#pragma unroll
  for (int c = 0; c < kChunkWaves; ++c) {
    l[c] = s[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (c <= w) {
      Parts kk, qk;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        bf16x8v f[KP];
#pragma unroll
        for (int p = 0; p < KP; ++p) f[p] = lds8(&lds.keys[p][K_::at(c * 16 + l16, m * 32 + q * 8)]);
        kk.add(f, kf[m]);
        qk.add(f, qf[m]);
      }
      l[c] = kk.sum();
      s[c] = qk.sum();
    }
  }
  const float ci = lds.cum[i], li = lds.low[i], bi = lds.beta[i];
  __syncthreads();                               // the keys are read: L takes their place
#pragma unroll
  for (int c = 0; c < kChunkWaves; ++c)
    if (c <= w) {
      const int j0 = c * 16 + q * 4;
      const f32x4 cj = *(const f32x4 *)&lds.cum[j0], lj = *(const f32x4 *)&lds.low[j0];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma clang fp reassociate(off)
        const float e = fast_exp2((ci - cj[r]) + (li - lj[r]));
        l[c][r] = j0 + r < i ? bi * e * l[c][r] : 0.0f;
        s[c][r] = j0 + r <= i ? a.scale * e * s[c][r] : 0.0f;
        if (!finite(l[c][r])) {
          atomicMin(&lds.first, i);
          l[c][r] = 0.0f;
        }
      }
      *(f32x4 *)&lds.L[i * kMatrixRow + j0] = l[c];
      if (!PIECES) map.P[map_tile(w, c)][lane] = s[c];
    }
  if (PIECES)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      if (m <= w / 2) {
        float e[8] = {s[2 * m][0], s[2 * m][1], s[2 * m][2], s[2 * m][3], s[2 * m + 1][0], s[2 * m + 1][1], s[2 * m + 1][2], s[2 * m + 1][3]};
        bf16x8v p[3];
        planes8(e, p);
#pragma unroll
        for (int n = 0; n < 3; ++n) map.pieces[map_piece(w, m)][n][lane] = __builtin_bit_cast(u32x4v, p[n]);
      }
  // The wave's own block on the diagonal: its rows were written by the wave itself.
  auto wave_fence = [] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  wave_fence();
  {
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = r == l16 ? 1.0f : 0.0f;
#pragma unroll
      for (int s = 0; s < r; ++s) x[r] = __builtin_fmaf(-lds.L[(w * 16 + r) * kMatrixRow + w * 16 + s], x[s], x[r]);
    }
    wave_fence();
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (r / 4 == q) lds.L[(w * 16 + r) * kMatrixRow + w * 16 + l16] = x[r];
  }
  __syncthreads();
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  auto put_block = [&](int rb, int cb, f32x4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) lds.L[(rb * 16 + q * 4 + r) * kMatrixRow + cb * 16 + l16] = -v[r];
  };
  if (w < 2) {
    const int b = 2 * w;
    const f32x4 x = mul_block(block_left(lds.L, b + 1, b, l16, q), block_right(lds.L, b, b, l16, q), zero);
    const f32x4 y = mul_block(block_left(lds.L, b + 1, b + 1, l16, q), x, zero);
    wave_fence();
    put_block(b + 1, b, y);
  }
  __syncthreads();
  {
    const int rb = 2 + w / 2, cb = w % 2;
    auto corner = [&](int s) {
      f32x4 y = mul_block(block_left(lds.L, s, 1, l16, q), block_right(lds.L, 1, cb, l16, q), zero);
      if (cb == 0) y = mul_block(block_left(lds.L, s, 0, l16, q), block_right(lds.L, 0, 0, l16, q), y);
      return y;
    };
    f32x4 y = mul_block(block_left(lds.L, rb, 2, l16, q), corner(2), zero);
    if (rb == 3) y = mul_block(block_left(lds.L, 3, 3, l16, q), corner(3), y);
    __syncthreads();                             // L's blocks there are read
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
      if (2 * m + s <= w) v = *(const f32x4 *)&lds.L[i * kMatrixRow + m * 32 + s * 16 + q * 4];
#pragma unroll
      for (int r = 0; r < 4; ++r) e[4 * s + r] = v[r];
    }
    bf16x8v p[3];
    planes8(e, p);
#pragma unroll
    for (int n = 0; n < 3; ++n) map.T[map_piece(w, m)][n][lane] = __builtin_bit_cast(u32x4v, p[n]);
  }
  if (tid == 0) map.gates[kRest][1] = __builtin_bit_cast(float, lds.first);
}

// The sequence of a workgroup and its columns' place.  The longest sequences come first (up to 64 of them: a
// lane each), so that the last workgroups to start are short; workgroups go to the eight XCDs in turn, and
// neighbouring columns, which read the same keys, to one of them.
__device__ __forceinline__ int nth_longest(const int32_t *off, int S, int n) {
  if (S > 64) return n;
  const int lane = (int)threadIdx.x & 63;
  const int length = lane < S ? off[lane + 1] - off[lane] : -1;
  int rank = 0;
  for (int j = 0; j < S; ++j) {
    const int other = __builtin_amdgcn_readlane(length, j);
    rank += other > length || (other == length && j < lane);
  }
  return __builtin_ctzll(__ballot(lane < S && rank == n));
}
__device__ __forceinline__ int column_of(int64_t unit, int columns) {
  const int c = (int)(unit % columns);
  return columns % 8 == 0 ? c % 8 * (columns / 8) + c / 8 : c;
}

// Products of planes, the largest part last: which plane of a and of b.
template <int A, int B> struct PlanePairs {
  static constexpr int kCount = A == 1 ? B : 6;
  static __device__ __forceinline__ constexpr int left(int i) { return A == 1 ? 0 : i == 0 || i == 3 ? 0 : i == 1 ? 1 : i == 2 ? 2 : i == 4 ? 1 : 0; }
  static __device__ __forceinline__ constexpr int right(int i) { return A == 1 ? B - 1 - i : i == 0 ? 2 : i == 1 ? 1 : i == 2 ? 0 : i == 3 ? 1 : 0; }
};

// Four consecutive elements of a row of outputs; whole where rows are aligned to four.
template <typename T> __device__ __forceinline__ bool packed_rows(const void *p, int64_t ld) {
  return ld % 4 == 0 && ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0;
}
template <typename T> __device__ __forceinline__ void store_four(T *p, const f32x4 &y, bool packed) {
  const float v[4] = {y[0], y[1], y[2], y[3]};
  if (packed) {
    Pack<T, 4>::store(p, v);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = from_float<T>(v[r]);
  }
}

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

// Rows of K elements in LDS, one after another, as copies straight from memory leave them; their
// 16-byte pieces are exchanged so that the rows and pieces that the hardware serves together lie in
// different banks (see Rows).
template <int K> struct Packed {
  static constexpr int kPieces = K / 8;
  static __device__ __forceinline__ int place(int row, int piece) {
    return piece ^ (kPieces == 16 ? row & 15 : kPieces == 8 ? row >> 1 & 7 : -(row >> 2) & 3);
  }
  static __device__ __forceinline__ int at(int row, int e) { return row * K + place(row, e >> 3) * 8 + (e & 7); }
};

template <typename T, int K> struct ChunkLds {
  static constexpr int KP = kKeyPlanes<T>;
  typedef Packed<K> K_;
  alignas(1024) unsigned short keys[KP][kChunk * K];
  alignas(1024) unsigned short queries[KP][kChunk * K];
  alignas(1024) u32x4v inverse[kMapPieces][3][64];
  alignas(1024) u32x4v scores[kMapPieces][3][64];
  alignas(1024) float gates[kGates][kChunk];
};

// A wave has 16 columns of the state (value channels) for all tokens and keys of its head, so
// what one product leaves is the next one's operand in the same lane and nothing goes
// between waves; keys, queries, T and P are shared in LDS.
//
// 8,192 tokens of 16 prompts, 32 heads of 128 by 128: 157 us.  The matrix units are busy 35% of it, the vector units (planes of S,
// R and U) 42%, two workgroups a CU, which is what 222 registers and 71 KB of LDS admit.  32 columns a wave halve the reads
// of LDS but leave one workgroup a CU: 382 us against 260 of an earlier form.
template <typename T, int K, bool WIDE>
__global__ void __launch_bounds__(kChunkThreads, sizeof(T) == 2 ? 2 : 1) chunk_walk_kernel(cortex_delta_t a, int32_t *status, const ChunkMap *maps) {
  typedef ChunkLds<T, K> Lds;
  constexpr int KP = Lds::KP, M = K / 32;
  constexpr int kItems = kChunk * (K / 8) / kChunkThreads;     // eights of keys that a thread brings in
  __shared__ Lds lds;
  const int failed = entry_status(status);
  const int64_t unit = blockIdx.x;
  const int tid = (int)threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, l16 = lane & 15;
  const int V = a.value_dim, wide = 16 * kChunkWaves, slices = (V + wide - 1) / wide, columns = a.heads * slices;
  const int seq = nth_longest(a.seq_offsets, a.num_seqs, (int)(unit / columns)), column = column_of(unit, columns), head = column / slices;
  const int v0 = column % slices * wide + w * 16;
  const bool works = v0 < V;
  const int g = head / (a.heads / a.key_heads);
  // (the same in every lane, and the compiler is told so)
  const int begin = __builtin_amdgcn_readfirstlane(a.seq_offsets[seq]), end = __builtin_amdgcn_readfirstlane(a.seq_offsets[seq + 1]);
  if (begin < 0 || end < begin || end > a.num_tokens) return;
  int pool = -1;
  if (a.state_in || a.state_out) {
    pool = state_row(a.state_index, seq, a.state_rows, status);
    if (pool < -1) return;
  }
  if (__syncthreads_or(failed != 0)) return;
  // column l16; of the state's tile 2 m + s the lane has entries 32 m + 8 q + 4 s .. + 3
  const int col = works ? v0 + l16 : 0;
  const int64_t state_at = (((int64_t)pool * a.heads + head) * V + col) * K + q * 8;
  f32x4 S[2 * M];
#pragma unroll
  for (int s = 0; s < 2 * M; ++s)
      S[s] = a.state_in && pool >= 0 && works ? *(const f32x4 *)(a.state_in + state_at + s / 2 * 32 + s % 2 * 4)
                                                 : f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const ChunkMap *map = maps + ((int64_t)(begin / kChunk) + seq) * a.heads + head;
  const T *ks = (const T *)a.k + g * K, *qs = (const T *)a.q + g * K;
  const T *vs = (const T *)a.v + (int64_t)head * V + col;
  T *ys = (T *)a.y + (int64_t)head * V + (works ? v0 + q * 4 : 0);
  const bool packed = packed_rows<T>(a.y, a.y_ld);
  // T, P, gates and queries of the next chunk are on their way while the state is updated, straight into LDS; its
  // keys meanwhile in registers, since the update reads this chunk's.  Rows past the sequence's end repeat its
  // last; places in a chunk are 32 bits (the host admits no longer rows).
  constexpr bool kStraight = KP == 1 && WIDE;    // bf16 in whole 16-byte pieces
  constexpr int kCopies = kMapPieces * 3 * 2, kRows = 512 / K;
  static_assert(kCopies % kChunkWaves == 0 && sizeof(ChunkMap) == (kCopies + 1) * 1024, "copies of 1 KB, the gates' last");
  Eight<T> kr[kItems], qr[kStraight ? 1 : kItems];
  auto bring = [&](int t0, const ChunkMap *map) {
    const int last = min(kChunk, end - t0) - 1;
#pragma unroll
    for (int i = 0; i < kCopies / kChunkWaves; ++i) {
      const int c = w * (kCopies / kChunkWaves) + i;
      copy_to_lds(map, (uint32_t)(c * 1024 + lane * 16), lds_place(lds.inverse) + (uint32_t)c * 1024);
    }
    if (w == 0) copy_to_lds(map, (uint32_t)(kCopies * 1024 + lane * 16), lds_place(lds.gates));
    const T *k0 = ks + (int64_t)t0 * a.k_ld, *q0 = qs + (int64_t)t0 * a.q_ld;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kChunkThreads + tid;
      const uint32_t row = min(id / (K / 8), last), o = id % (K / 8) * 8;
      kr[i].template load<WIDE>(k0 + (row * (uint32_t)a.k_ld + o));
      if constexpr (!kStraight) qr[i].template load<WIDE>(q0 + (row * (uint32_t)a.q_ld + o));
    }
    if constexpr (kStraight)
#pragma unroll
      for (int i = 0; i < kChunk / kRows / kChunkWaves; ++i) {
        const int first = (w * (kChunk / kRows / kChunkWaves) + i) * kRows, row = first + lane / (K / 8);
        const uint32_t e = (uint32_t)Lds::K_::place(row, lane % (K / 8)) * 8, r = (uint32_t)min(row, last);
        copy_to_lds(q0, (r * (uint32_t)a.q_ld + e) * 2, lds_place(lds.queries) + (uint32_t)(first * K * 2));
      }
  };
  if (begin < end) bring(begin, map);
#pragma unroll 1
  for (int t0 = begin; t0 < end; t0 += kChunk) {
    const int last = min(kChunk, end - t0) - 1;
    copies_done<0>();
    __syncthreads();                             // the last chunk's keys are read
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int id = i * kChunkThreads + tid, at = Lds::K_::at(id / (K / 8), id % (K / 8) * 8);
      bf16x8v f[KP];
      kr[i].planes(f);
#pragma unroll
      for (int p = 0; p < KP; ++p) *(u32x4v *)&lds.keys[p][at] = __builtin_bit_cast(u32x4v, f[p]);
      if constexpr (!kStraight) {
        qr[i].planes(f);
#pragma unroll
        for (int p = 0; p < KP; ++p) *(u32x4v *)&lds.queries[p][at] = __builtin_bit_cast(u32x4v, f[p]);
      }
    }
    T v[4][4];
    const T *vt = vs + (int64_t)t0 * a.v_ld;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) v[t][r] = vt[(uint32_t)min(t * 16 + q * 4 + r, last) * (uint32_t)a.v_ld];
    __syncthreads();                             // keys, queries, T, P and gates are there
    const float decay = lds.gates[kRest][0];
    int first = __builtin_bit_cast(int, lds.gates[kRest][1]);
    auto to_planes = [](const f32x4 &lo, const f32x4 &hi, bf16x8v (&p)[3]) {
      float e[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      planes8(e, p);
    };
    f32x4 kS[4], y[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) kS[t] = y[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf16x8v sp[3];
      to_planes(S[2 * m], S[2 * m + 1], sp);
      typedef PlanePairs<KP, 3> Pairs;
      auto by_state = [&](const unsigned short (&rows)[KP][kChunk * K], f32x4 (&to)[4], auto turned) {
        bf16x8v f[4][KP];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int p = 0; p < KP; ++p) f[t][p] = lds8(&rows[p][Lds::K_::at(t * 16 + l16, m * 32 + q * 8)]);
#pragma unroll
        for (int i = 0; i < Pairs::kCount; ++i)
#pragma unroll
          for (int t = 0; t < 4; ++t)
            to[t] = turned ? mfma_bf16x32(sp[Pairs::right(i)], f[t][Pairs::left(i)], to[t]) : mfma_bf16x32(f[t][Pairs::left(i)], sp[Pairs::right(i)], to[t]);
      };
      by_state(lds.keys, kS, std::false_type());
      by_state(lds.queries, y, std::true_type());
    }
    typedef PlanePairs<3, 3> Pairs;
    // c += pieces of T or P by the planes of 64 tokens; turned, a token is the result's column
    auto by_map = [&](const u32x4v (&map)[kMapPieces][3][64], const bf16x8v (&p)[2][3], f32x4 (&to)[4], auto turned) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 2 * m; t < 4; t += 2) {
          bf16x8v f[2][3];
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 3; ++i) f[s][i] = __builtin_bit_cast(bf16x8v, map[map_piece(t + s, m)][i][lane]);
#pragma unroll
          for (int i = 0; i < Pairs::kCount; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s)
              to[t + s] = turned ? mfma_bf16x32(p[m][Pairs::right(i)], f[s][Pairs::left(i)], to[t + s])
                                 : mfma_bf16x32(f[s][Pairs::left(i)], p[m][Pairs::right(i)], to[t + s]);
        }
    };
    f32x4 u[4];
    bf16x8v planes[2][3];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const f32x4 beta = *(const f32x4 *)&lds.gates[kBeta][t * 16 + q * 4], grow = *(const f32x4 *)&lds.gates[kGrow][t * 16 + q * 4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = beta[r] * (to_float<T>(v[t][r]) - grow[r] * kS[t][r]);
        kS[t][r] = t * 16 + q * 4 + r <= last ? x : 0.0f;
      }
      y[t] *= a.scale * lds.gates[kGrow][t * 16 + l16];
      u[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    drop_odd(kS, q, first);
#pragma unroll
    for (int m = 0; m < 2; ++m) to_planes(kS[2 * m], kS[2 * m + 1], planes[m]);
    by_map(lds.inverse, planes, u, std::false_type());
    drop_odd(u, q, first);
#pragma unroll
    for (int m = 0; m < 2; ++m) to_planes(u[2 * m], u[2 * m + 1], planes[m]);
    by_map(lds.scores, planes, y, std::true_type());
#pragma unroll
    for (int t = 0; t < 4; ++t) u[t] *= *(const f32x4 *)&lds.gates[kWeight][t * 16 + q * 4];
#pragma unroll
    for (int m = 0; m < 2; ++m) to_planes(u[2 * m], u[2 * m + 1], planes[m]);
    // y, before the copies that the next chunk waits for: four columns of a token a lane
    T *yt = ys + (int64_t)t0 * a.y_ld;
    if (__any(first < kChunk))
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int from = __shfl(first, q * 4 + r);
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (t * 16 + l16 >= from) y[t][r] = __builtin_nanf("");
      }
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (works && t * 16 + l16 <= last) store_four<T>(yt + (uint32_t)(t * 16 + l16) * (uint32_t)a.y_ld, y[t], packed);
    __syncthreads();                             // all but the keys is read
    if (t0 + kChunk < end) {
      map += a.heads;
      bring(t0 + kChunk, map);
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf16x8v kt[2][2][KP];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        S[2 * m + s] *= decay;
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
            S[2 * m + s] = mfma_bf16x32(kt[s][h][KeyPairs::left(i)], planes[h][KeyPairs::right(i)], S[2 * m + s]);
    }
    if (first < kChunk)
#pragma unroll
      for (int s = 0; s < 2 * M; ++s) S[s] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
  }
  if (a.state_out && pool >= 0 && works)
#pragma unroll
    for (int s = 0; s < 2 * M; ++s) *(f32x4 *)(a.state_out + state_at + s / 2 * 32 + s % 2 * 4) = S[s];
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
  alignas(16) f32x4 U[2][4][64];
  alignas(16) f32x4 V[2][4][64];
  alignas(16) unsigned short keys[KP][kChunk * K_::kStride];
  alignas(1024) u32x4v inverse[2][kMapPieces][3][64];
  alignas(1024) f32x4 scores[2][kMapTiles][64];
  alignas(16) float gates[2][kGates][kChunk];
  alignas(16) int first[2][16];
};

// The same for few columns: eight waves share 16 of them, so that the chain from one state to
// the next is short.  Four waves of 16 tokens each form it: keys by state, R; U; the
// next state, with an LDS exchange and a barrier between.  Four more bring in values and gates and form the
// outputs beside them, those of a chunk while the next one's R is made.  One more brings T and P into LDS.
//
// PART 0: whole sequences.  Where even these are few, a sequence is cut into segments of Q tokens: what
// a segment does to the state that enters it is S M + N, and part 1 finds N (from a zero state) and M
// (from the unit rows, without values) as columns of their own, V + K of them; enter_segments_kernel
// joins them; part 2 forms the outputs from the state that enters.
//
// The latency of a chunk bounds it: 2 us at 128 by 128, 1.5 of them the chain's three exchanges (32,768 tokens of 32 heads, a
// workgroup a CU: 1,140 us for 512 chunks; matrix units busy 23%, LDS 34%).  Without the outputs' stores it took 0.3 us a chunk
// less, which is why a lane stores four columns at once (1,222 us in all before, 1,171 since); values loaded so as well changed
// nothing.
template <typename T, int K, int PART, bool WIDE>
__global__ void __launch_bounds__(kChainThreads) chunk_chain_kernel(cortex_delta_t a, int32_t *status, const ChunkMap *maps, float *segments, float *nowhere, int Q) {
  typedef ChainLds<T, K> Lds;
  constexpr int KP = Lds::KP, M = Lds::M;
  constexpr int ST = K == 128 ? 2 : 1;           // tiles of 16 state entries of a wave
  __shared__ Lds lds;
  const int failed = entry_status(status);
  const int64_t unit = blockIdx.x;
  const int tid = (int)threadIdx.x, lane = tid & 63, q = lane >> 4, l16 = lane & 15;
  // the tokens of a wave; the products of T and of P grow with them, so that a SIMD's two waves have five tiles together
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), w = wave < kChunkWaves ? wave : kChunkWaves - 1 - wave % kChunkWaves;
  const int V = a.value_dim, rows = PART == 0 ? V : V + K, slices = (PART == 1 ? rows : V) / 16, columns = a.heads * slices;
  const int place = (int)(unit / columns), slot = PART == 0 ? nth_longest(a.seq_offsets, a.num_seqs, place) : place;
  const int column = column_of(unit, columns), head = column / slices, v0 = column % slices * 16;
  const bool values = PART != 1 || v0 < V;       // else unit rows
  const int g = head / (a.heads / a.key_heads);
  int seq = slot, begin, end, first, last_token;
  if constexpr (PART == 0) {
    first = begin = a.seq_offsets[seq];
    last_token = end = a.seq_offsets[seq + 1];
    if (begin < 0 || end < begin || end > a.num_tokens) return;
  } else {
    const Chunk c = find_chunk(a.seq_offsets, a.num_seqs, a.num_tokens, Q, slot);
    if (c.seq < 0) return;
    seq = c.seq;
    begin = c.begin;
    end = c.end;
    first = c.first;
    last_token = c.last;
    if (PART == 1 && end == last_token) return;  // nothing follows it
  }
  // (the same in every lane, and the compiler is told so)
  begin = __builtin_amdgcn_readfirstlane(begin);
  end = __builtin_amdgcn_readfirstlane(end);
  first = __builtin_amdgcn_readfirstlane(first);
  seq = __builtin_amdgcn_readfirstlane(seq);
  int pool = -1;
  if (PART != 1 && (a.state_in || a.state_out)) {
    pool = state_row(a.state_index, seq, a.state_rows, status);
    if (pool < -1) return;
  }
  if (__syncthreads_or(failed != 0)) return;
  const ChunkMap *const first_map = maps + ((int64_t)(first / kChunk) + seq + (begin - first) / kChunk) * a.heads + head;
  // What a chunk needs is loaded as soon as the last chunk's is used up, without a condition, so
  // that nothing waits for it: the last chunk repeats its own.  Rows past the sequence's end
  // repeat its last.  Places in a chunk are 32 bits (the host admits no longer rows).
  Eight<T> raw[M];
  uint32_t own = 0;
  auto load_own = [&](const T *rows) {
#pragma unroll
    for (int m = 0; m < M; ++m) raw[m].template load<WIDE>(rows + own + m * 32);
  };
  auto last_of = [&](int t0) { return min(kChunk, end - t0) - 1; };
  auto after = [&](int t0) { return t0 + kChunk < end ? t0 + kChunk : t0; };
  if (wave == 2 * kChunkWaves) {
    // T and P of the next chunk go straight into LDS, 1 KB at a time
    static_assert(offsetof(ChunkMap, P) == kMapPieces * 3 * 1024, "P follows T");
    auto bring = [&](const ChunkMap *map, int b) {
#pragma unroll
      for (int i = 0; i < kMapPieces * 3 + (PART == 1 ? 0 : kMapTiles); ++i)
        copy_to_lds(map, (uint32_t)(i * 1024 + lane * 16),
                    i < kMapPieces * 3 ? lds_place(lds.inverse[b]) + i * 1024 : lds_place(lds.scores[b]) + (i - kMapPieces * 3) * 1024);
    };
    const ChunkMap *map = first_map;
    int b = 0;
    if (begin < end) bring(map, 0);
    for (int t0 = begin; t0 < end; t0 += kChunk, b ^= 1) {
      copies_done<0>();
      __syncthreads();
      __syncthreads();                           // the outputs of the last chunk, which read the other buffer, are formed
      if (t0 + kChunk < end) {
        map += a.heads;
        bring(map, b ^ 1);
      }
      __syncthreads();
    }
    return;
  }
  if (wave >= kChunkWaves) {
    if (begin >= end) return;
    const T *qs = (const T *)a.q + g * K + q * 8, *vs = (const T *)a.v + (int64_t)head * V + (values ? v0 : 0) + l16;
    T *ys = (T *)a.y + (int64_t)head * V + v0 + q * 4;
    const bool packed = packed_rows<T>(a.y, a.y_ld);
    T v[4];
    float gate;
    auto load_values = [&](int t0, const ChunkMap *of) {
      const T *vt = vs + (int64_t)t0 * a.v_ld;
      const int last = last_of(t0);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = values ? vt[(uint32_t)min(w * 16 + q * 4 + r, last) * (uint32_t)a.v_ld] : (T)0.0f;
      gate = of->gates[w][lane];
    };
    auto load_queries = [&](int t0) {
      own = (uint32_t)min(w * 16 + l16, last_of(t0)) * (uint32_t)a.q_ld;
      load_own(qs + (int64_t)t0 * a.q_ld);
    };
    auto put_values = [&](int b) {
      lds.V[b][w][lane] = f32x4{to_float<T>(v[0]), to_float<T>(v[1]), to_float<T>(v[2]), to_float<T>(v[3])};
      lds.gates[b][w][lane] = gate;
      if (w == kRest) {
        const int first = __builtin_bit_cast(int, __shfl(gate, 1));
        if (lane < 16) lds.first[b][lane] = first;
      }
    };
    const ChunkMap *map = first_map;
    // the first chunk's values and gates; then the second's are on their way
    load_values(begin, map);
    if (PART != 1) load_queries(begin);
    put_values(0);
    int coming = after(begin);
    if (coming != begin) map += a.heads;
    load_values(coming, map);
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
    // y of the chunk from t0 on, of buffer b, once its updates are there: P by U in float32 on both
    // sides as they stand, k = 4 q + step of each 16 tokens.  A lane ends with four columns of a token.
    auto finish = [&](int b) {
      f32x4 yp[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
      for (int c = 0; c < kChunkWaves; ++c)
        if (c <= w) yp[c % 2] = mul_block(lds.U[b][c][lane], lds.scores[b][map_tile(w, c)][lane], yp[c % 2]);
      y += yp[0] + yp[1];
    };
    auto store = [&](int t0, int b) {
      typedef int i32x4 __attribute__((ext_vector_type(4)));
      const i32x4 from = *(const i32x4 *)&lds.first[b][q * 4];
      const int i = w * 16 + l16;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (i >= from[r]) y[r] = __builtin_nanf("");
      // Without a condition, so that the wait for a later load does not take the stores with it (they may not have
      // been made): rows past the end go where nothing is read.
      T *const p = i <= last_of(t0) ? ys + (int64_t)t0 * a.y_ld + (uint32_t)i * (uint32_t)a.y_ld : (T *)nowhere + l16 * 4;
      store_four<T>(p, y, packed);
    };
    int t0 = begin, b = 0;
#pragma unroll 1
    for (;; b ^= 1) {
      __syncthreads();                           // the state, values and gates are there
      if (PART != 1 && t0 != begin) finish(b ^ 1);
      __syncthreads();                           // R and the keys are there
      if (PART != 1 && t0 != begin) store(t0 - kChunk, b ^ 1);
      const int next = after(t0);
      if constexpr (PART != 1) {
        // beside U; the next state comes after it
        Parts qp;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          bf16x8v qf[KP], s[3];
          raw[m].planes(qf);
#pragma unroll
          for (int p = 0; p < 3; ++p) s[p] = __builtin_bit_cast(bf16x8v, lds.S[p][m][lane]);
          qp.add(s, qf);
        }
        y = qp.sum() * (lds.gates[b][kGrow][w * 16 + l16] * a.scale);
        load_queries(next);
      }
      __syncthreads();                           // U is there
      put_values(b ^ 1);
      coming = after(next);
      if (coming != next) map += a.heads;
      load_values(coming, map);
      if (next == t0) break;
      t0 = next;
    }
    if (PART != 1) {
      finish(b);
      store(t0, b);
    }
    return;
  }
  __builtin_amdgcn_s_setprio(2);                 // the outputs have time until the next state
  // the wave's part of the state: 32 entries m, its halves of four in eight from `half` on
  const int sm = K == 128 ? w : K == 64 ? w / 2 : 0, half = K == 128 ? 0 : K == 64 ? w % 2 : w;
  const bool holds = K > 32 || w < 2;
  const int entry = sm * 32 + q * 8 + half * 4;  // and four further on for the second tile
  const int64_t state_at = (((int64_t)pool * a.heads + head) * V + v0 + l16) * K + entry;
  float *const segment = PART == 0 ? nullptr : segments + (((int64_t)slot * a.heads + head) * rows + v0 + l16) * K + entry;
  f32x4 S[ST];
  auto put_state = [&]() {
    if (!holds) return;
#pragma unroll
    for (int s = 0; s < ST; ++s) put_planes4(&lds.S[0][sm][0], M * 64, lane, half + s, S[s]);
  };
#pragma unroll
  for (int s = 0; s < ST; ++s)
  {
    S[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (PART == 0 && a.state_in && pool >= 0 && holds) S[s] = *(const f32x4 *)(a.state_in + state_at + s * 4);
    if (PART == 2 && holds) S[s] = *(const f32x4 *)(segment + s * 4);
    if (PART == 1 && !values)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[s][r] = v0 - V + l16 == entry + s * 4 + r ? 1.0f : 0.0f;
  }
  put_state();
  const T *ks = (const T *)a.k + g * K + q * 8;
  // Values of the lane's tokens that are not finite become 0: their products with the zeros above
  // the diagonal would carry them to earlier tokens.  The first is noted.
  auto drop = [&](f32x4 &x, int b) {
#pragma clang fp reassociate(off)
    const float none = (x[0] * 0.0f + x[1] * 0.0f) + (x[2] * 0.0f + x[3] * 0.0f);
    if (!__any(none != 0.0f)) return;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!finite(x[r])) {
        atomicMin(&lds.first[b][l16], w * 16 + q * 4 + r);
        x[r] = 0.0f;
      }
  };
  if (begin < end) {
    own = (uint32_t)min(w * 16 + l16, last_of(begin)) * (uint32_t)a.k_ld;
    load_own(ks + (int64_t)begin * a.k_ld);
  }
  int b = 0;
#pragma unroll 1
  for (int t0 = begin; t0 < end; t0 += kChunk, b ^= 1) {
    const int last = last_of(t0);
    const int next = after(t0);
    __syncthreads();                             // the state, values and gates are there; the last chunk's keys are read
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
    const f32x4 beta = *(const f32x4 *)&lds.gates[b][kBeta][w * 16 + q * 4], grow = *(const f32x4 *)&lds.gates[b][kGrow][w * 16 + q * 4];
    f32x4 x = beta * (lds.V[b][w][lane] - grow * kp.sum());
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (w * 16 + q * 4 + r > last) x[r] = 0.0f;
    drop(x, b);
    put_planes4(&lds.R[0][w / 2][0], 2 * 64, lane, w % 2, x);
    own = (uint32_t)min(w * 16 + l16, last_of(next)) * (uint32_t)a.k_ld;
    load_own(ks + (int64_t)next * a.k_ld);
    __syncthreads();                             // R and the keys are there
    Parts up;
#pragma unroll
    for (int m = 0; m < 2; ++m)
      if (m <= w / 2) {
        bf16x8v t[3], s[3];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          t[p] = __builtin_bit_cast(bf16x8v, lds.inverse[b][map_piece(w, m)][p][lane]);
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
    drop(u, b);
    put_planes4(&lds.W[0][w / 2][0], 2 * 64, lane, w % 2, u * *(const f32x4 *)&lds.gates[b][kWeight][w * 16 + q * 4]);
    if (PART != 1) lds.U[b][w][lane] = u;
    __syncthreads();                             // U is there
    if (holds) {
      const bool gone = lds.first[b][l16] < kChunk;
      const float decay = lds.gates[b][kRest][0];
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
        S[s] = S[s] * decay + sp[s].sum();
        if (gone) S[s] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
      }
    }
    put_state();
  }
  float *const to = PART == 1 ? segment : a.state_out && pool >= 0 && end == last_token ? a.state_out + state_at : nullptr;
  if (to && holds)
#pragma unroll
    for (int s = 0; s < ST; ++s) *(f32x4 *)(to + s * 4) = S[s];
}

// The states that enter a sequence's segments, in the place of what they add: s <- s M + N.  A workgroup
// takes 16 rows of a head's state; a wave K / 4 of their entries (float32 matrix units, k = 4 q + step of each
// 16 on both sides), M's loads for the next segment on their way.  About 1.5 us a segment, its loads' latency.
template <int K>
__global__ void __launch_bounds__(kChunkThreads) enter_segments_kernel(cortex_delta_t a, int32_t *status, float *segments, int Q) {
  constexpr int kRow = K + 4, kTiles = K < 64 ? 1 : K / 64, kBlocks = K / 16;
  __shared__ __attribute__((aligned(16))) float lds[2][16 * kRow];
  const int failed = entry_status(status);
  const int tid = (int)threadIdx.x, lane = tid & 63, w = tid >> 6, q = lane >> 4, l16 = lane & 15;
  const int V = a.value_dim, v0 = (int)blockIdx.x % (V / 16) * 16, head = (int)blockIdx.x / (V / 16) % a.heads;
  const int seq = (int)blockIdx.x / (V / 16) / a.heads;
  const int begin = a.seq_offsets[seq], end = a.seq_offsets[seq + 1];
  if (begin < 0 || end < begin || end > a.num_tokens) return;
  int pool = -1;
  if (a.state_in || a.state_out) {
    pool = state_row(a.state_index, seq, a.state_rows, status);
    if (pool < -1) return;
  }
  if (__syncthreads_or(failed != 0)) return;
  const bool works = w * kTiles * 16 < K;
  const int k0 = works ? w * kTiles * 16 : 0;    // the wave's entries
  const int64_t stride = (int64_t)a.heads * (V + K) * K;
  float *at = segments + ((int64_t)(begin / Q + seq) * a.heads + head) * (V + K) * K;
  // a lane has rows 4 q .. + 3 of entry l16 of each tile
  f32x4 s[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      s[t][r] = a.state_in && pool >= 0 ? a.state_in[(((int64_t)pool * a.heads + head) * V + v0 + q * 4 + r) * K + k0 + t * 16 + l16] : 0.0f;
  float m[kTiles][kBlocks][4];
  f32x4 add[kTiles];
  auto load = [&]() {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) m[t][b][i] = at[(int64_t)(V + b * 16 + q * 4 + i) * K + k0 + t * 16 + l16];
#pragma unroll
      for (int r = 0; r < 4; ++r) add[t][r] = at[(int64_t)(v0 + q * 4 + r) * K + k0 + t * 16 + l16];
    }
  };
  int64_t t0 = begin;
  int b = 0;
#pragma unroll 1
  for (;; b ^= 1) {
    const bool more = t0 + Q < end;
    if (more && works) load();
    if (works)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          at[(int64_t)(v0 + q * 4 + r) * K + k0 + t * 16 + l16] = s[t][r];
          lds[b][(q * 4 + r) * kRow + k0 + t * 16 + l16] = s[t][r];
        }
    if (!more) return;
    __syncthreads();
    if (works) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) s[t] = add[t];
#pragma unroll
      for (int c = 0; c < kBlocks; ++c) {
        const f32x4 left = *(const f32x4 *)&lds[b][l16 * kRow + c * 16 + q * 4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s[t] = mul_block(left, f32x4{m[t][c][0], m[t][c][1], m[t][c][2], m[t][c][3]}, s[t]);
      }
    }
    at += stride;
    t0 += Q;
  }
}

}  // namespace cortex
