// What the sequence operators share: element types, the chunks into which the
// prompts of a batch are cut, the pool rows of their states, and the gate and
// step-size functions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cortex_device.hpp"
#include "cortex_host.hpp"

namespace cortex {

typedef __bf16 bf16_t;

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }
// Rounds to nearest even, as the hardware conversion does.
template <typename T> __device__ __forceinline__ T from_float(float v) { return (T)v; }

// V consecutive elements as one load or store where the address allows it
// (V elements of 16 bytes together), else element by element (V = 1).
template <typename T, int V> struct Pack {
  typedef T type __attribute__((ext_vector_type(V)));
  static __device__ __forceinline__ void load(const T *p, float (&v)[V]) {
    const type q = *(const type *)p;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_float<T>(q[i]);
  }
  static __device__ __forceinline__ void store(T *p, const float (&v)[V]) {
    type q;
#pragma unroll
    for (int i = 0; i < V; ++i) q[i] = from_float<T>(v[i]);
    *(type *)p = q;
  }
};
template <typename T> struct Pack<T, 1> {
  static __device__ __forceinline__ void load(const T *p, float (&v)[1]) { v[0] = to_float<T>(*p); }
  static __device__ __forceinline__ void store(T *p, const float (&v)[1]) { *p = from_float<T>(v[0]); }
};

// 16 bytes a lane straight into LDS, lane after lane from `to` on.  The compiler does not
// see the load: the caller waits for it (copies_done) before the barrier.
// `base` and `to` are the same in every lane.
__device__ __forceinline__ void copy_to_lds(const void *base, uint32_t offset, uint32_t to) {
  const uint64_t at = (uint64_t)base;
  const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 |
                           (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(offset),
               "s"(uniform)
               : "memory", "m0");
}
template <int N> __device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }
__device__ __forceinline__ uint32_t lds_place(const void *p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

// The status as earlier launches left it, through the caches: these kernels have
// many waves, and none of them waits for another launch's word.
__device__ __forceinline__ int entry_status(const int32_t *status) {
  return __hip_atomic_load(status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

constexpr float kLog2e = 1.44269504088896340736f;

// v_exp_f32: 2^x to one unit in the last place, denormal results flushed to zero.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// A decay's rate to the base 2.  Past the float range it stays a number, so that a step
// of 0, as tokens past a sequence's end have it, keeps the state (0 * infinity would not).
__device__ __forceinline__ float decay_rate(float A) {
  constexpr float kLowest = -3.402823466e38f;
  const float r = A * kLog2e;
  return r < kLowest ? kLowest : r;              // (a NaN stays one)
}

// v / (1 + exp(-v)).
__device__ __forceinline__ float silu(float v) {
  return v * __builtin_amdgcn_rcpf(1.0f + fast_exp2(v * -kLog2e));
}

__device__ __forceinline__ float sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + fast_exp2(v * -kLog2e));
}

// softplus(v) = max(v, 0) + log1p(e), e = exp(-|v|) in (0, 1].  With
// s = e / (2 + e) <= 1/3, log1p(e) = 2 atanh(s) = 2 s (1 + s^2/3 + s^4/5 + ...);
// after the s^14 term what is left is below 2^-27 of the sum.  log(1 + e) itself
// would lose the small step sizes: at dt = 0.001 it is off by 6e-5 of the value.
__device__ __forceinline__ float softplus(float v) {
  const float e = fast_exp2(-kLog2e * __builtin_fabsf(v));
  const float s = e * __builtin_amdgcn_rcpf(2.0f + e);
  const float q = s * s;
  float p = 1.0f / 15.0f;
  p = __builtin_fmaf(p, q, 1.0f / 13.0f);
  p = __builtin_fmaf(p, q, 1.0f / 11.0f);
  p = __builtin_fmaf(p, q, 1.0f / 9.0f);
  p = __builtin_fmaf(p, q, 1.0f / 7.0f);
  p = __builtin_fmaf(p, q, 1.0f / 5.0f);
  p = __builtin_fmaf(p, q, 1.0f / 3.0f);
  p = __builtin_fmaf(p, q, 1.0f);
  const float r = __builtin_fmaf(2.0f * s, p, __builtin_fmaxf(v, 0.0f));
  return v != v ? v : r;      // fmax drops a NaN
}

__device__ __forceinline__ float step_size(const cortex_scan_t &a, float raw, float bias) {
  const float v = raw + bias;
  return a.softplus ? softplus(v) : v;
}

// v of the lane that a data-parallel shift names; `none` in lanes that it leaves out.
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ float shifted(float v, float none) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL,
                                                               ROWS, 0xf, false));
}

// Inclusive combination over the lanes of a wave, neutral element e: from 1, 2, 4
// and 8 lanes below in a row of 16, lane 15 to the row above, lane 31 to the upper half.
// HALVES: over each half of the wave.
template <bool HALVES, typename F> __device__ __forceinline__ float lane_prefix(float v, float e, F f) {
  v = f(v, shifted<0x111>(v, e));
  v = f(v, shifted<0x112>(v, e));
  v = f(v, shifted<0x114>(v, e));
  v = f(v, shifted<0x118>(v, e));
  v = f(v, shifted<0x142, 0xa>(v, e));
  if (!HALVES) v = f(v, shifted<0x143, 0xc>(v, e));
  return v;
}
__device__ __forceinline__ float lane_sums(float v) {
  return lane_prefix<false>(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float half_sums(float v) {
  return lane_prefix<true>(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float last_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_sum(float v) { return last_lane(lane_sums(v)); }
__device__ __forceinline__ float wave_max(float v) {
  return last_lane(lane_prefix<false>(v, -__builtin_inff(), [](float a, float b) { return __builtin_fmaxf(a, b); }));
}

// ---------------------------------------------------------------------------
// Chunks.  Sequence i is cut into chunks of Q tokens from its own first token
// on.  Its chunks take the slots from off[i] / Q + i on: that is at least as
// many as it needs (an empty sequence gets one too), so a grid of T / Q + S
// slots serves any lengths, and a slot finds its sequence by a search over the
// offsets alone, with no table to build first.
// ---------------------------------------------------------------------------
struct Chunk {
  int seq;            // -1: the slot is unused, or its sequence's offsets are broken
  int first, last;    // the sequence's rows
  int begin, end;     // the chunk's rows
  int slot0;          // the sequence's first slot
};

__host__ __device__ inline int64_t chunk_slots(int64_t T, int64_t S, int Q) { return T / Q + S; }

// The largest i in [0, S) with off[i] / Q + i <= slot, by a search that splits
// the range 64 ways a round, one offset per lane (one round up to 64 sequences).
// It ends and stays inside [0, S) whatever the offsets hold.
__device__ __forceinline__ int seq_of_slot(const int32_t *off, int S, int Q, int slot) {
  const int lane = (int)(threadIdx.x & 63);
  int lo = 0, hi = S;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6;
    const int64_t i = lo + (int64_t)lane * step;
    const bool below = i < hi && off[i] / Q + i <= slot;
    const int n = __builtin_popcountll(__ballot(below));
    const int64_t nlo = lo + (int64_t)(n > 0 ? n - 1 : 0) * step;
    const int64_t nhi = nlo + step;
    lo = (int)nlo;
    hi = nhi < hi ? (int)nhi : hi;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Every slot below S checks one pair of offsets, so a batch's are all checked.
__device__ __forceinline__ void check_offsets(const int32_t *off, int S, int T, int slot, int32_t *status) {
  if (slot >= S) return;
  const int a = off[slot], b = off[slot + 1];
  if (a < 0 || b < a || b > T || (slot == 0 && a != 0) || (slot == S - 1 && b != T))
    raise_status(status, CORTEX_ST_SEQ_OFFSETS);
}

__device__ __forceinline__ Chunk find_chunk(const int32_t *off, int S, int T, int Q, int slot) {
  Chunk c;
  c.seq = seq_of_slot(off, S, Q, slot);
  c.first = off[c.seq];
  c.last = off[c.seq + 1];
  c.slot0 = c.first / Q + c.seq;
  const int64_t begin = (int64_t)c.first + (int64_t)(slot - c.slot0) * Q;
  const bool fine = c.first >= 0 && c.first <= c.last && c.last <= T && slot >= c.slot0 &&
                    (begin < c.last || slot == c.slot0);
  if (!fine) {
    c.seq = -1;
    return c;
  }
  c.begin = (int)begin;
  c.end = c.last - c.begin > Q ? c.begin + Q : c.last;
  return c;
}

// Pool row of sequence i's state, -1 for none; -2 where the index is out of
// range, which it reports.
__device__ __forceinline__ int state_row(const int32_t *index, int i, int rows, int32_t *status) {
  const int r = index ? index[i] : i;
  if (r < -1 || r >= rows) {
    raise_status(status, CORTEX_ST_INPUT_RANGE);
    return -2;
  }
  return r;
}

// Between the launches of a prompt that is split over its length (scan.hip).
struct SegmentScratch {
  float *state;      // [slots, D, N]: a segment's result from zero, then the state that enters it
  float *steps;      // [slots, channels or heads]: its sum of dt
};

// Workgroups go to the eight XCDs in turn.  Each XCD takes a run of neighbouring
// units, so that those which read the same rows find them in the L2 that they share.
__device__ __forceinline__ int64_t unit_of_block(int64_t units) {
  const int64_t per = (units + 7) / 8;
  return (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8;
}
inline unsigned blocks_of_units(int64_t units) { return (unsigned)((units + 7) / 8 * 8); }

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Grids count tiles of channels in 16 bits.
constexpr int32_t kMaxChannels = 1 << 18;
// 64 rows of elements stay below 2^31, so that places in a sub-chunk take 32 bits.
constexpr int64_t kMaxRowStride = 1 << 25;

// Host checks that the prompt and step forms share: sizes of the batch.
inline bool bad_batch(int32_t dtype, int32_t S, int32_t T, int32_t channels, int32_t state_rows, const int32_t *index,
                      bool has_state) {
  if (dtype != CORTEX_F32 && dtype != CORTEX_BF16) return true;
  if (S < 0 || T < 0 || channels < 1 || channels > kMaxChannels || state_rows < 0) return true;
  // slots of chunks are counted in 32 bits
  if ((int64_t)S + T > 0x7fff0000) return true;
  return has_state && !index && state_rows < S;
}

}  // namespace cortex
