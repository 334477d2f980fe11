// Norms of queries and keys per head, their weights and their rotation, in one pass.
//
// Every element is read once and written once: the bytes bound it (8,192 tokens of 40 heads of 128 bf16, 168 MB: 33 us, 5.1
// TB/s, what a large copy reaches).  A rotation
// pairs elements R / 2 apart or neighbours, so a lane takes two pieces of 16 bytes
// whose pairs are all its own, and a head's lanes (a power of two of them, some
// without work where the head is none) only have to add their squares.  A wave
// takes heads of one token, 64 / lanes of them at a time, so that a token's cosines
// and sines are made once by the wave, an angle a lane, and held in registers.
#include "sequence.hpp"

namespace cortex {

constexpr int kNormWaves = 4;
constexpr int kMaxHeadDim = 512;

// cos and sin of position * freq, turned into turns and cut to half a turn in 64
// bits: at position 2^31 the angle is off by 2^-22, at 200,000 by 2^-35.
__device__ __forceinline__ void angle(int position, float freq, float &c, float &s) {
  constexpr double kTurn = 0.15915494309189533577;
  double turns = (double)position * (double)freq * kTurn;
  turns -= __builtin_rint(turns);
  sincospif(2.0f * (float)turns, &s, &c);
}

// Where a token's head begins, in q or in k.
template <typename T> struct NormRow {
  const T *in;
  T *out;
  const float *weight;
};
template <typename T> __device__ __forceinline__ NormRow<T> norm_row(const cortex_qk_norm_t &a, int64_t t, int r) {
  const int P = a.head_dim;
  if (r < a.heads)
    return {(const T *)a.q + t * a.q_ld + (int64_t)r * P, (T *)a.q_out + t * a.q_out_ld + (int64_t)r * P, a.q_weight};
  r -= a.heads;
  return {(const T *)a.k + t * a.k_ld + (int64_t)r * P, (T *)a.k_out + t * a.k_out_ld + (int64_t)r * P, a.k_weight};
}

__device__ __forceinline__ float norm_scale(const cortex_qk_norm_t &a, float squares) {
  if (a.norm == CORTEX_NORM_NONE) return 1.0f;
  const float v = (a.norm == CORTEX_NORM_RMS ? squares / (float)a.head_dim : squares) + a.eps;
  return 1.0f / __builtin_sqrtf(v);
}

// Sum over 2^k neighbouring lanes, the same in each.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
  if (LANES > 1) v += shifted<0xb1>(v, 0.0f);
  if (LANES > 2) v += shifted<0x4e>(v, 0.0f);
  if (LANES > 4) v += shifted<0x141>(v, 0.0f);
  if (LANES > 8) v += shifted<0x140>(v, 0.0f);
  if (LANES > 16) v += __shfl_xor(v, 16);
  if (LANES > 32) v += __shfl_xor(v, 32);
  return v;
}

// Rows at 16-byte boundaries; LANES lanes a head.  A wave takes the rows (a
// token's heads, queries then keys) from `first` on, `rows` of them.
template <typename T, int LANES, bool INTERLEAVED>
__global__ void __launch_bounds__(64 * kNormWaves) norm_wide_kernel(cortex_qk_norm_t a, int32_t *status, int splits) {
  constexpr int V = 16 / (int)sizeof(T), kRound = 64 / LANES;
  __shared__ float turn[kNormWaves][2][kMaxHeadDim / 2];
  if (entry_status(status) != 0) return;
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int64_t task = (int64_t)blockIdx.x * kNormWaves + wave;
  const int64_t t = task / splits;
  if (t >= a.num_tokens) return;
  const int R = a.rotary_dim, P = a.head_dim, total = a.heads + a.key_heads;
  const int part = lane % LANES, group = lane / LANES;
  const bool works = part * 2 * V < P;
  // the lane's two pieces
  int lo = part * 2 * V, hi = lo + V;
  if (!INTERLEAVED && lo < R) {
    lo = part * V;
    hi = R / 2 + lo;
  }
  if (!works) lo = hi = 0;
  const bool turns = works && lo < R;            // halves: all of both pieces; neighbours: as far as R reaches
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    c[i] = 1.0f;
    s[i] = 0.0f;
  }
  if (R) {
    const int position = a.positions[t];
    for (int i = lane; i < R / 2; i += 64) angle(position, a.freqs[i], turn[wave][0][i], turn[wave][1][i]);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (turns)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int at = INTERLEAVED ? lo / 2 + i : lo + i;
        if (at < R / 2) {
          c[i] = turn[wave][0][at];
          s[i] = turn[wave][1][at];
        }
      }
  }
  const int each = (total + splits - 1) / splits, first = (int)(task % splits) * each, last = min(first + each, total);
  // Heads of q, then of k, each with their weights in registers.
  auto run = [&](const T *in, T *out, const float *weight, int from, int to) {
    if (from >= to) return;
    float g[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      g[i] = weight ? weight[lo + i] : 1.0f;
      g[V + i] = weight ? weight[hi + i] : 1.0f;
    }
    for (int r = from + group; r - group < to; r += kRound) {
      const T *p = in + (int64_t)min(r, to - 1) * P;
      float x[2][V], squares = 0.0f;
      Pack<T, V>::load(p + lo, x[0]);
      Pack<T, V>::load(p + hi, x[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < V; ++i) squares = __builtin_fmaf(x[h][i], x[h][i], squares);
      const float m = norm_scale(a, lanes_sum<LANES>(works ? squares : 0.0f));
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < V; ++i) x[h][i] *= m * g[h * V + i];
      float y[2][V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float *d = INTERLEAVED ? &y[2 * i / V][2 * i % V] : &y[0][i], *e = INTERLEAVED ? &y[2 * i / V][2 * i % V + 1] : &y[1][i];
        const float f = INTERLEAVED ? x[2 * i / V][2 * i % V] : x[0][i], k = INTERLEAVED ? x[2 * i / V][2 * i % V + 1] : x[1][i];
        // what is not rotated is left alone: a sine of 0 would carry an infinity or NaN to the other
        const bool turned = turns && (!INTERLEAVED || lo / 2 + i < R / 2);
        *d = turned ? f * c[i] - k * s[i] : f;
        *e = turned ? k * c[i] + f * s[i] : k;
      }
      if (works && r < to) {
        Pack<T, V>::store(out + (int64_t)r * P + lo, y[0]);
        Pack<T, V>::store(out + (int64_t)r * P + hi, y[1]);
      }
    }
  };
  run((const T *)a.q + t * a.q_ld, (T *)a.q_out + t * a.q_out_ld, a.q_weight, first, min(last, a.heads));
  run((const T *)a.k + t * a.k_ld, (T *)a.k_out + t * a.k_out_ld, a.k_weight, max(first - a.heads, 0), last - a.heads);
}

// Any alignment and any even sizes: a wave a head, pairs by lane.
template <typename T>
__global__ void __launch_bounds__(64 * kNormWaves) norm_pair_kernel(cortex_qk_norm_t a, int32_t *status) {
  constexpr int N = kMaxHeadDim / 128;
  if (entry_status(status) != 0) return;
  const int lane = (int)threadIdx.x & 63;
  const int total = a.heads + a.key_heads, R = a.rotary_dim, P = a.head_dim;
  const int64_t task = (int64_t)blockIdx.x * kNormWaves + (threadIdx.x >> 6), t = task / total;
  if (t >= a.num_tokens) return;
  const NormRow<T> row = norm_row<T>(a, t, (int)(task % total));
  float x[N], y[N], squares = 0.0f;
  int at[N], to[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int pair = n * 64 + lane;
    const bool halves = !a.interleaved && pair < R / 2;
    at[n] = halves ? pair : 2 * pair;
    to[n] = halves ? pair + R / 2 : 2 * pair + 1;
    x[n] = y[n] = 0.0f;
    if (pair < P / 2) {
      x[n] = to_float<T>(row.in[at[n]]);
      y[n] = to_float<T>(row.in[to[n]]);
    }
    squares = __builtin_fmaf(x[n], x[n], __builtin_fmaf(y[n], y[n], squares));
  }
  const float m = norm_scale(a, lanes_sum<64>(squares));
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int pair = n * 64 + lane;
    if (pair >= P / 2) continue;
    float u = x[n] * m, v = y[n] * m;
    if (row.weight) {
      u *= row.weight[at[n]];
      v *= row.weight[to[n]];
    }
    if (pair < R / 2) {
      float c, s;
      angle(a.positions[t], a.freqs[pair], c, s);
      const float turned = u * c - v * s;
      v = v * c + u * s;
      u = turned;
    }
    row.out[at[n]] = from_float<T>(u);
    row.out[to[n]] = from_float<T>(v);
  }
}

template <typename T, int LANES> int launch_wide(const cortex_qk_norm_t &a, int32_t *status, int splits, void *stream) {
  const int64_t tasks = (int64_t)a.num_tokens * splits;
  const unsigned grid = (unsigned)((tasks + kNormWaves - 1) / kNormWaves);
  const hipStream_t st = (hipStream_t)stream;
  if (a.interleaved) norm_wide_kernel<T, LANES, true><<<grid, 64 * kNormWaves, 0, st>>>(a, status, splits);
  else norm_wide_kernel<T, LANES, false><<<grid, 64 * kNormWaves, 0, st>>>(a, status, splits);
  return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T> int launch_norm(const cortex_qk_norm_t &a, int32_t *status, void *stream) {
  constexpr int V = 16 / (int)sizeof(T);
  auto rows16 = [](const void *p, int64_t ld) { return aligned16(p) && ld % V == 0; };
  const bool wide = a.head_dim % (2 * V) == 0 && (a.interleaved || a.rotary_dim % (2 * V) == 0) && rows16(a.q, a.q_ld) &&
                    rows16(a.q_out, a.q_out_ld) && (!a.key_heads || (rows16(a.k, a.k_ld) && rows16(a.k_out, a.k_out_ld)));
  const int total = a.heads + a.key_heads;
  const int64_t tasks = (int64_t)a.num_tokens * total;
  // A wave a head while there are at most four a SIMD: 1 token of 40 heads of 128 2.9 us against 4.0, 100 tokens 3.8
  // against 4.4, but 200 tokens 5.2 against 4.6 and 8,192 126 against 43.
  if (!wide || tasks <= 4096) {
    norm_pair_kernel<T><<<(unsigned)((tasks + kNormWaves - 1) / kNormWaves), 64 * kNormWaves, 0, (hipStream_t)stream>>>(a, status);
    return hipGetLastError() == hipSuccess ? CORTEX_OK : CORTEX_E_HIP;
  }
  int lanes = 1;
  while (lanes * 2 * V < a.head_dim) lanes *= 2;
  // A token's heads go to several waves as long as that leaves at most two a SIMD (1,024 of them): 512 tokens of 72
  // heads of 256 13.5 us with 4 waves each, 15.7 with 8, 18.8 with one; 8,192 of 40 heads of 128 43 with one, 65 with
  // ten.  Loads of two heads at once changed nothing (43.3, 15.6).
  const int at_once = 64 / lanes, most = (total + at_once - 1) / at_once;
  const int64_t want = 2048 / a.num_tokens;
  const int splits = (int)(want < 1 ? 1 : want < most ? want : most);
  switch (lanes) {
    case 1: return launch_wide<T, 1>(a, status, splits, stream);
    case 2: return launch_wide<T, 2>(a, status, splits, stream);
    case 4: return launch_wide<T, 4>(a, status, splits, stream);
    case 8: return launch_wide<T, 8>(a, status, splits, stream);
    case 16: return launch_wide<T, 16>(a, status, splits, stream);
    case 32: return launch_wide<T, 32>(a, status, splits, stream);
    default: return launch_wide<T, 64>(a, status, splits, stream);
  }
}

}  // namespace cortex

extern "C" int cortex_qk_norm(const cortex_qk_norm_t *a, int32_t *status, void *stream) {
  using namespace cortex;
  if (!a || !status) return CORTEX_E_INVAL;
  if (a->dtype != CORTEX_F32 && a->dtype != CORTEX_BF16) return CORTEX_E_INVAL;
  const int64_t P = a->head_dim;
  if (a->num_tokens < 0 || a->heads < 1 || a->key_heads < 0 || a->heads > 65536 || a->key_heads > 65536) return CORTEX_E_INVAL;
  if (P < 2 || P > kMaxHeadDim || P % 2 || a->rotary_dim < 0 || a->rotary_dim > P || a->rotary_dim % 2) return CORTEX_E_INVAL;
  if (a->norm < CORTEX_NORM_NONE || a->norm > CORTEX_NORM_L2 || !(a->eps >= 0.0f)) return CORTEX_E_INVAL;
  if (a->q_ld < a->heads * P || a->q_out_ld < a->heads * P) return CORTEX_E_INVAL;
  if (a->key_heads && (a->k_ld < a->key_heads * P || a->k_out_ld < a->key_heads * P)) return CORTEX_E_INVAL;
  // four waves a workgroup, at most a wave a token and head, and a grid has less than 2^32 threads
  if ((int64_t)a->num_tokens * (a->heads + a->key_heads) >= (int64_t)1 << 25) return CORTEX_E_INVAL;
  if (a->num_tokens == 0) return CORTEX_OK;
  if (!a->q || !a->q_out || (a->key_heads && (!a->k || !a->k_out)) || (a->rotary_dim && (!a->positions || !a->freqs)))
    return CORTEX_E_INVAL;
  return a->dtype == CORTEX_BF16 ? launch_norm<bf16_t>(*a, status, stream) : launch_norm<float>(*a, status, stream);
}
