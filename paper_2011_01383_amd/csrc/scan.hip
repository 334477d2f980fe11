// Selective state space scan, for prompts and for single tokens.
#include "scan_head.hpp"
#include "scan_head32.hpp"
#include "sequence.hpp"

#include <algorithm>

namespace cortex {

constexpr int kScanWave = 64;

// N consecutive floats (N a multiple of 4, 16-byte aligned).
template <int N> __device__ __forceinline__ void load_floats(const float *p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 q = *(const float4 *)(p + i);
    v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
  }
}
template <int N> __device__ __forceinline__ void store_floats(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *(float4 *)(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}

// ---------------------------------------------------------------------------
// Splitting a prompt over its length.  The recurrence of a state entry is
// linear, h <- a h + b, so a segment of tokens acts on the state that enters it
// as h <- (product of its a) h + (its result from a zero state); the product of
// exp(dt A) is exp(A sum dt).  Three launches: every segment's result and step
// sum from zero (part 1), the states that enter the segments, one after another
// (enter_kernel), then the outputs from those (part 2).  With enough sequences
// and channels to fill the GPU, or few tokens, one launch walks each sequence
// whole (part 0): half the arithmetic.
// ---------------------------------------------------------------------------
// One thread per state entry walks its sequence's segments.
template <bool HEAD>
__global__ void __launch_bounds__(256) enter_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w, int Q) {
  constexpr int U = 8;                           // segments loaded ahead of the chain through them
  if (entry_status(status) != 0) return;
  const int seq = (int)blockIdx.y;
  const int first = a.seq_offsets[seq], last = a.seq_offsets[seq + 1];
  if (first < 0 || last < first || last > a.num_tokens) return;
  const int row = a.state_in || a.state_out ? state_row(a.state_index, seq, a.state_rows, status) : -1;
  if (row < -1) return;
  const int64_t per_slot = (int64_t)a.channels * a.state_size;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= per_slot) return;
  const int d = (int)(e / a.state_size), k = HEAD ? d / a.head_dim : d;
  const int rates = HEAD ? a.channels / a.head_dim : a.channels;
  const float A2 = decay_rate(a.A[HEAD ? k : e]);
  float h = row >= 0 && a.state_in ? a.state_in[row * per_slot + e] : 0.0f;
  const int count = (last - first + Q - 1) / Q;
  const int64_t slot0 = first / Q + seq;
  float *st = w.state + slot0 * per_slot + e;
  const float *sd = w.steps + slot0 * rates + k;
  for (int c = 0; c < count; c += U) {
    float r[U], f[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int j = c + i < count ? c + i : count - 1;
      r[i] = st[j * per_slot];
      f[i] = fast_exp2(A2 * sd[(int64_t)j * rates]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (c + i < count) {
        st[(c + i) * per_slot] = h;
        h = __builtin_fmaf(h, f[i], r[i]);
      }
  }
  if (row >= 0 && a.state_out) a.state_out[row * per_slot + e] = h;
}

// ---------------------------------------------------------------------------
// Decays per channel, prompts: a lane is a channel and keeps its N states in
// registers.  The exponentials bound it: N of them and 4 N products and sums
// for every channel and token.  B and C of kTile tokens are the same for the
// whole wave: it keeps them in LDS as floats and reads them by broadcast.  What
// the next kAhead tokens (of B and C: the next tile) need is loaded while these
// are worked on.
//
// 32,768 tokens of 2,048 channels and 16 states, split: 266 us (part 1) + 19 (the
// states between) + 309 (part 2), traced.  That is 260 and 302 ns of a SIMD a token
// and wave, for 100 and 138 vector instructions: about 218 and 292 ns at 1.9 ns each
// and 3.5 for an exponential, as four waves a SIMD of nothing else take for them.
// ---------------------------------------------------------------------------
constexpr int kAhead = 4, kTile = 16;

template <typename T, int N, int PART>
__global__ void __launch_bounds__(kScanWave) channel_scan_kernel(cortex_scan_t a, int32_t *status, SegmentScratch w, int Q) {
  if (entry_status(status) != 0) return;
  const int slot = (int)blockIdx.x, g = (int)blockIdx.z;
  const bool checks = blockIdx.y == 0 && g == 0;
  int seq, begin, end;
  if constexpr (PART == 0) {
    seq = slot;
    if (checks) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, seq, status);
    begin = a.seq_offsets[seq];
    end = a.seq_offsets[seq + 1];
    if (begin < 0 || end < begin || end > a.num_tokens) return;
  } else {
    if (PART == 1 && checks) check_offsets(a.seq_offsets, a.num_seqs, a.num_tokens, slot, status);
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
  const int per_group = a.channels / a.groups;
  const int lane = (int)threadIdx.x, tile0 = (int)blockIdx.y * kScanWave;
  const bool active = tile0 + lane < per_group;
  // lanes past the group's last channel repeat it and store nothing
  const int d = g * per_group + (active ? tile0 + lane : per_group - 1);

  float h[N], A2[N];
  const int64_t state_at = ((int64_t)(PART == 0 ? row : slot) * a.channels + d) * N;
  if (PART == 2) load_floats<N>(w.state + state_at, h);
  else if (PART == 0 && row >= 0 && a.state_in) load_floats<N>(a.state_in + state_at, h);
  else
#pragma unroll
    for (int n = 0; n < N; ++n) h[n] = 0.0f;
#pragma unroll
  for (int n = 0; n < N; ++n) A2[n] = decay_rate(a.A[(int64_t)d * N + n]);
  const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f, skip = a.skip ? a.skip[d] : 0.0f;
  const T *xs = (const T *)a.x + d, *ds = (const T *)a.dt + d, *zs = (const T *)a.z + d;
  T *ys = (T *)a.y + d;
  const T *Bs = (const T *)a.B + g * N, *Cs = (const T *)a.C + g * N;
  const bool gate = a.z != nullptr;
  float steps = 0.0f;

  constexpr int kShared = PART == 1 ? N : 2 * N;              // B, and C after it
  constexpr int kStage = kTile * kShared / kScanWave;
  __shared__ float shared_bc[kTile][kShared];
  T x0[kAhead], d0[kAhead], z0[kAhead], bc0[kStage];
  auto fetch = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t t = t0 + i < end ? t0 + i : end - 1;
      x0[i] = xs[t * a.x_ld];
      d0[i] = ds[t * a.dt_ld];
      if (PART != 1 && gate) z0[i] = zs[t * a.z_ld];
    }
  };
  auto fetch_bc = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kStage; ++i) {
      const int e = i * kScanWave + lane, k = e % kShared;
      const int64_t t = t0 + e / kShared < end ? t0 + e / kShared : end - 1;
      bc0[i] = k < N ? Bs[t * a.B_ld + k] : Cs[t * a.C_ld + k - N];
    }
  };
  if (begin < end) {
    fetch(begin);
    fetch_bc(begin);
  }
  for (int tile = begin; tile < end; tile += kTile) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kStage; ++i) (&shared_bc[0][0])[i * kScanWave + lane] = to_float<T>(bc0[i]);
    __syncthreads();
    if (tile + kTile < end) fetch_bc(tile + kTile);
    const int stop = end - tile < kTile ? end : tile + kTile;
#pragma unroll 1
    for (int t0 = tile; t0 < stop; t0 += kAhead) {
      float x[kAhead], dt[kAhead], z[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        x[i] = to_float<T>(x0[i]);
        dt[i] = step_size(a, to_float<T>(d0[i]), bias);
        z[i] = to_float<T>(z0[i]);
      }
      if (t0 + kAhead < end) fetch(t0 + kAhead);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t t = t0 + i;
        if (t < stop) {
          const float u = dt[i] * x[i];
          const float *B = shared_bc[t - tile], *C = B + N;
          float y = skip * x[i];
#pragma unroll
          for (int n = 0; n < N; ++n) {
            h[n] = __builtin_fmaf(h[n], fast_exp2(dt[i] * A2[n]), u * B[n]);
            if (PART != 1) y = __builtin_fmaf(h[n], C[n], y);
          }
          if (PART == 1) {
            steps += dt[i];
          } else if (active) {
            if (gate) y *= silu(z[i]);
            ys[t * a.y_ld] = from_float<T>(y);
          }
        }
      }
    }
  }
  if (!active) return;
  if (PART == 1) {
    store_floats<N>(w.state + state_at, h);
    w.steps[(int64_t)slot * a.channels + d] = steps;
  }
  if (PART == 0 && row >= 0 && a.state_out) store_floats<N>(a.state_out + state_at, h);
}

// ---------------------------------------------------------------------------
// One token.  N / 4 lanes share a channel, each with four neighbouring states,
// so a wave reads and writes whole lines of the state, which bounds it: 8 bytes
// a state entry against 5 operations.  A lane takes U channels of a head, which
// share B and C, or U rows of a channel, which share its decays; their loads are
// on their way together.  The new state is stored past the caches (nontemporal:
// 134 MB of states 70 -> 66 us).  Loads past them pay where the states were not
// in the 256 MB last-level cache (67 MB: 40 -> 32 us, 134 MB: 70 -> 59, the states
// of other layers used in between) and cost where they were (134 MB: 48 -> 58,
// 67 MB: 28 -> 30, 34 MB: 16 -> 19, one layer again and again), so they are taken
// from 64 MiB on, where a model's layers no longer fit together.  Measured: 256
// rows of 2,048 channels and 16 states (71 MB) 14 us, 5.2 TB/s; 64 rows of 4,096
// and 128 (268 MB) 60 us, 4.5 TB/s.
// ---------------------------------------------------------------------------
constexpr int kStepThreads = 256;

template <typename T, int N, bool HEAD, int U, bool STREAM>
__global__ void __launch_bounds__(kStepThreads) scan_step_kernel(cortex_scan_t a, int32_t *status) {
  constexpr int L = N / 4, kChannels = kStepThreads / L;         // lanes per channel, channels side by side
  constexpr int UC = HEAD ? U : 1, UR = HEAD ? 1 : U;            // channels and rows of a lane
  if (entry_status(status) != 0) return;
  const int part = (int)(threadIdx.x % L), c0 = (int)blockIdx.y * kChannels * UC;
  const int b0 = (int)blockIdx.x * UR;
  typedef T vec4 __attribute__((ext_vector_type(4)));
  int row[UR];
#pragma unroll
  for (int r = 0; r < UR; ++r) {
    row[r] = -1;
    if (a.state_in || a.state_out) {
      row[r] = b0 + r < a.num_seqs ? state_row(a.state_index, b0 + r, a.state_rows, status) : -1;
      if (row[r] < -1) return;
    }
  }
  // channel u / UR and row u % UR; past the last it repeats that and stores nothing
  f32x4 h[U];
  float x[U], raw[U], z[U];
  vec4 Bv[U], Cv[U];
  int d[U], b[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    d[u] = min(c0 + u / UR * kChannels + (int)(threadIdx.x / L), a.channels - 1);
    b[u] = min(b0 + u % UR, a.num_seqs - 1);
    const int slot = row[u % UR];
    h[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (slot >= 0 && a.state_in) {
      const f32x4 *p = (const f32x4 *)(a.state_in + ((int64_t)slot * a.channels + d[u]) * N + part * 4);
      h[u] = STREAM ? __builtin_nontemporal_load(p) : *p;
    }
    const int64_t t = b[u];
    x[u] = to_float<T>(((const T *)a.x)[t * a.x_ld + d[u]]);
    raw[u] = to_float<T>(((const T *)a.dt)[t * a.dt_ld + (HEAD ? d[u] / a.head_dim : d[u])]);
    if (a.z) z[u] = to_float<T>(((const T *)a.z)[t * a.z_ld + d[u]]);
    const int g = d[u] / (a.channels / a.groups);
    const T *B = (const T *)a.B + t * a.B_ld + g * N + part * 4, *C = (const T *)a.C + t * a.C_ld + g * N + part * 4;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      Bv[u][n] = B[n];
      Cv[u][n] = C[n];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = HEAD ? d[u] / a.head_dim : d[u];
    const bool stores = c0 + u / UR * kChannels + (int)(threadIdx.x / L) < a.channels && b0 + u % UR < a.num_seqs;
    const float dt = step_size(a, raw[u], a.dt_bias ? a.dt_bias[k] : 0.0f);
    const float w = dt * x[u], decay = HEAD ? fast_exp2(dt * decay_rate(a.A[k])) : 0.0f;
    float y = 0.0f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const float f = HEAD ? decay : fast_exp2(dt * decay_rate(a.A[(int64_t)k * N + part * 4 + n]));
      h[u][n] = __builtin_fmaf(h[u][n], f, w * to_float<T>(Bv[u][n]));
      y = __builtin_fmaf(h[u][n], to_float<T>(Cv[u][n]), y);
    }
    const int slot = row[u % UR];
    if (slot >= 0 && a.state_out && stores)
      __builtin_nontemporal_store(h[u], (f32x4 *)(a.state_out + ((int64_t)slot * a.channels + d[u]) * N + part * 4));
#pragma unroll
    for (int m = 1; m < L; m <<= 1) y += __shfl_xor(y, m);
    if (part == 0 && stores) {
      if (a.skip) y = __builtin_fmaf(a.skip[k], x[u], y);
      if (a.z) y *= silu(z[u]);
      ((T *)a.y)[(int64_t)b[u] * a.y_ld + d[u]] = from_float<T>(y);
    }
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// Tokens of a segment, 0 for one launch over whole sequences.
//
// The host knows how many tokens and sequences there are, not how long each is, so
// a rule can be right for equal lengths, for a ramp of them, or for one long prompt
// among short ones, not for all.  Times in us, split and in one launch.
//
// Per channel.  A wave is bound by its arithmetic, which a split doubles; in one
// launch the longest sequence is a chain of tokens at 0.45 us each (N = 16).  The
// switch is where equal lengths lose by the split what a ramp gains, one wave a SIMD
// (1,024): 8,192 tokens of 2,048 bf16 channels, 24 prompts: equal 167 and 163, ramp
// 172 and 302; 32: 164 and 124, 177 and 231; 64: 174 and 84, 205 and 156.  With fewer
// channels and shorter prompts it would be lower (4,096 float32 tokens of 512
// channels, 64 prompts: 51 and 34, 52 and 62; 100: 61 and 25, 60 and 41), but a long
// prompt among them would then cost ten times a split.  Up to 36 tokens three
// launches cost more than any chain (32 tokens: 20 and 17, 48: 20 and 24; N = 64: 44 and
// 44, 44 and 64).  Segments are as long as leaves four waves a SIMD (8,192 tokens of 16
// sequences and 2,048 channels, 64 tokens: 158 equal, 169 ramp; 128: 200; 32: 143, 150, but
// with twice the states between the passes; one sequence of 32,768 tokens, 256: 537; 512: 746;
// 128: 497); below half a wave a SIMD they go down to 16 (257 tokens of 512 float32
// channels, 16 tokens: 22; 24: 27; 32: 32; 64: 56).
//
// Per head.  A unit is 64 channels of a head in one sequence.  In one launch the
// longest sequence is a chain of sub-chunks at 1.6 to 2.4 us (float32 3.3 to 5.2).  8,192
// tokens of 32 bf16 heads, N = 128: 8 prompts (256 units): equal 126 and 85, ramp 133
// and 144, half of the tokens in one prompt 131 and 320; 12 (384): 138 and 77, 145 and
// 116, 159 and 315; 15 (480): 142 and 65, 145 and 97, 166 and 320; 16,384 tokens of 64
// heads, 7 prompts (448): 436 and 255, 397 and 380; 4,096 float32 tokens of 16 heads, 24
// prompts (384): 67 and 37, 70 and 59.  At 400 units the most that either choice loses is
// about the same.  Short prompts: 192 tokens of one unit 16 and 16, of 32 (N = 128) 24 and
// 20; 256: 16 and 19, 24 and 25; 64 units: 256: 35 and 25, 512: 43 and 44; 128 units of four
// sequences, half of the tokens in one: 512: 43 and 25, 1,024: 47 and 45; float32, 16 units:
// 128: 20 and 18, 192: 21 and 25.  The workgroups that the GPU holds at once (three a CU at
// N = 128, four below) get a segment each, of at least 64 tokens: 32,768 tokens of 64 heads,
// 2,752 tokens: 561; 1,024: 575; 256: 669; 4,099 float32 tokens of 16 heads, 96 tokens: 49;
// 64: 56; 256: 70.
constexpr int64_t kWholeUnits = 400, kWholeWaves = 1024;   // from these on one launch
static int segment_tokens(int64_t T, int64_t S, int64_t D, int N, int head_dim) {
  int64_t Q;
  if (head_dim) {
    const int64_t groups = D / head_dim * ((head_dim + 63) / 64), units = S * groups;
    if (units >= kWholeUnits || T <= 160 + 2 * units) return 0;
    const int64_t segments = (N == 128 ? 768 : 1024) / groups;
    Q = ((T + segments - 1) / segments + 31) / 32 * 32;
    if (Q < 64) Q = 64;
  } else {
    const int64_t tiles = (D + kScanWave - 1) / kScanWave;
    if (S * tiles >= kWholeWaves || T <= 36) return 0;
    Q = 256;
    while (Q > 32 && T / Q * tiles < 4096) Q /= 2;
    if (T / Q * tiles < 512) Q = 16;
  }
  return T <= Q ? 0 : (int)Q;                    // one segment is not split
}

// A call that does not split has to bring a workspace too, of 256 bytes.
static size_t scratch_bytes(int64_t slots, int64_t D, int N) {
  return std::max<size_t>(256, (size_t)slots * D * (N + 1) * sizeof(float));
}

// The most slots that segment_tokens leads to for up to T tokens in up to S sequences
// (more of either may mean fewer: longer segments, or one launch).  A batch that is
// split has less than kWholeUnits / groups sequences.  Per head T / Q is at most T / 64 and
// at most `segments`.  Per channel Q = 256 gives T / 256; a smaller one was taken since
// T / 2Q * tiles < 4,096 (for 16: T / 32 * tiles < 512), so T / Q <= 2 * (4,095 / tiles) + 1.
static int64_t most_slots(int64_t T, int64_t S, int64_t D, int N, int head_dim) {
  if (head_dim) {
    const int64_t groups = D / head_dim * ((head_dim + 63) / 64);
    const int64_t segments = (N == 128 ? 768 : 1024) / groups;
    if (groups >= kWholeUnits || segments < 2 || T <= 160 + 2 * groups) return 0;
    return std::min(T / 64, segments) + std::min(S, (kWholeUnits - 1) / groups);
  }
  const int64_t tiles = (D + kScanWave - 1) / kScanWave;
  if (tiles >= kWholeWaves || T <= 36) return 0;
  return std::min(T / 16, std::max(T / 256, 2 * (4095 / tiles) + 1)) + std::min(S, (kWholeWaves - 1) / tiles);
}

static SegmentScratch scratch_of(const cortex_scan_t &a, int Q, void *ws) {
  SegmentScratch w = {nullptr, nullptr};
  if (Q) {
    w.state = (float *)ws;
    w.steps = w.state + (size_t)chunk_slots(a.num_tokens, a.num_seqs, Q) * a.channels * a.state_size;
  }
  return w;
}

static bool launched() { return hipGetLastError() == hipSuccess; }

template <typename T, int N> int launch_channel(const cortex_scan_t &a, int32_t *status, void *ws, void *stream) {
  const int Q = segment_tokens(a.num_tokens, a.num_seqs, a.channels, N, 0);
  const SegmentScratch w = scratch_of(a, Q, ws);
  const unsigned tiles = (a.channels / a.groups + kScanWave - 1) / kScanWave;
  const hipStream_t st = (hipStream_t)stream;
  if (!Q) {
    channel_scan_kernel<T, N, 0><<<dim3(a.num_seqs, tiles, a.groups), kScanWave, 0, st>>>(a, status, w, 0);
    return launched() ? CORTEX_OK : CORTEX_E_HIP;
  }
  const unsigned slots = (unsigned)chunk_slots(a.num_tokens, a.num_seqs, Q);
  const unsigned entries = (unsigned)(((int64_t)a.channels * N + 255) / 256);
  channel_scan_kernel<T, N, 1><<<dim3(slots, tiles, a.groups), kScanWave, 0, st>>>(a, status, w, Q);
  if (!launched()) return CORTEX_E_HIP;
  enter_kernel<false><<<dim3(entries, a.num_seqs), 256, 0, st>>>(a, status, w, Q);
  if (!launched()) return CORTEX_E_HIP;
  channel_scan_kernel<T, N, 2><<<dim3(slots, tiles, a.groups), kScanWave, 0, st>>>(a, status, w, Q);
  return launched() ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T, int N, int PART>
int launch_head_part(const cortex_scan_t &a, int32_t *status, const SegmentScratch &w, int Q, unsigned slots, hipStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);         // elements of 16 bytes
  auto rows16 = [](const void *p, int64_t ld) { return aligned16(p) && ld % V == 0; };
  const bool wide = rows16(a.x, a.x_ld) && rows16(a.B, a.B_ld) && rows16(a.C, a.C_ld) && rows16(a.z, a.z ? a.z_ld : 0) &&
                    rows16(a.y, a.y_ld);
  const int64_t units = (int64_t)slots * (a.channels / a.head_dim) * ((a.head_dim + 63) / 64);
  const unsigned grid = blocks_of_units(units);
  if constexpr (sizeof(T) == 2) {
    if (wide) head_mfma_kernel<N, PART, true><<<grid, kHeadThreads, 0, st>>>(a, status, w, Q, units);
    else head_mfma_kernel<N, PART, false><<<grid, kHeadThreads, 0, st>>>(a, status, w, Q, units);
  } else {
    if (wide) head_mfma32_kernel<N, PART, true><<<grid, kHeadThreads, 0, st>>>(a, status, w, Q, units);
    else head_mfma32_kernel<N, PART, false><<<grid, kHeadThreads, 0, st>>>(a, status, w, Q, units);
  }
  return launched() ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T, int N> int launch_head(const cortex_scan_t &a, int32_t *status, void *ws, void *stream) {
  const int Q = segment_tokens(a.num_tokens, a.num_seqs, a.channels, N, a.head_dim);
  const SegmentScratch w = scratch_of(a, Q, ws);
  const hipStream_t st = (hipStream_t)stream;
  if (!Q) return launch_head_part<T, N, 0>(a, status, w, 0, a.num_seqs, st);
  const unsigned slots = (unsigned)chunk_slots(a.num_tokens, a.num_seqs, Q);
  const unsigned entries = (unsigned)(((int64_t)a.channels * N + 255) / 256);
  const int rc = launch_head_part<T, N, 1>(a, status, w, Q, slots, st);
  if (rc != CORTEX_OK) return rc;
  enter_kernel<true><<<dim3(entries, a.num_seqs), 256, 0, st>>>(a, status, w, Q);
  if (!launched()) return CORTEX_E_HIP;
  return launch_head_part<T, N, 2>(a, status, w, Q, slots, st);
}

template <typename T, int N, bool HEAD, int U, bool STREAM>
int launch_step_units(const cortex_scan_t &a, int32_t *status, void *stream) {
  constexpr int kRows = HEAD ? 1 : U, kChannels = kStepThreads / (N / 4) * (HEAD ? U : 1);
  scan_step_kernel<T, N, HEAD, U, STREAM><<<dim3((a.num_seqs + kRows - 1) / kRows, (a.channels + kChannels - 1) / kChannels),
                                            kStepThreads, 0, (hipStream_t)stream>>>(a, status);
  return launched() ? CORTEX_OK : CORTEX_E_HIP;
}

// Two of a lane's units while that leaves eight waves a SIMD (four: 134 MB of
// states 76 us, two: 70, eight: 98).
template <typename T, int N, bool HEAD> int launch_step(const cortex_scan_t &a, int32_t *status, void *stream) {
  const int64_t entries = (int64_t)a.num_seqs * a.channels * N;
  if (entries / 4 / 64 < 2 * 8192) return launch_step_units<T, N, HEAD, 1, false>(a, status, stream);
  return entries < (16 << 20) ? launch_step_units<T, N, HEAD, 2, false>(a, status, stream)
                              : launch_step_units<T, N, HEAD, 2, true>(a, status, stream);
}

static bool bad_scan_size(int32_t channels, int32_t groups, int32_t state_size, int32_t head_dim) {
  const int N = state_size;
  if (channels < 1 || groups < 1 || channels % groups) return true;
  if (head_dim == 0) return N != 8 && N != 16 && N != 32 && N != 64;
  if (head_dim < 16 || head_dim > 256 || head_dim % 16 || (channels / groups) % head_dim) return true;
  return N != 16 && N != 32 && N != 64 && N != 128;
}

static int check_scan(const cortex_scan_t *a, bool step, int32_t *status) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (bad_batch(a->dtype, a->num_seqs, a->num_tokens, a->channels, a->state_rows, a->state_index,
                a->state_in || a->state_out))
    return CORTEX_E_INVAL;
  if (bad_scan_size(a->channels, a->groups, a->state_size, a->head_dim) || a->groups > 65535) return CORTEX_E_INVAL;
  if (step ? a->num_tokens != a->num_seqs : !a->seq_offsets) return CORTEX_E_INVAL;
  const int64_t dts = a->head_dim ? a->channels / a->head_dim : a->channels;
  const int64_t bc = (int64_t)a->groups * a->state_size;
  const int64_t most = kMaxRowStride;
  if (a->x_ld > most || (a->z && a->z_ld > most) || a->y_ld > most || a->dt_ld > most || a->B_ld > most || a->C_ld > most)
    return CORTEX_E_INVAL;
  if (a->x_ld < a->channels || a->y_ld < a->channels || a->dt_ld < dts || a->B_ld < bc || a->C_ld < bc ||
      (a->z && a->z_ld < a->channels))
    return CORTEX_E_INVAL;
  if (!a->A || !aligned16(a->state_in) || !aligned16(a->state_out)) return CORTEX_E_INVAL;
  if (a->num_tokens > 0 && (!a->x || !a->dt || !a->B || !a->C || !a->y)) return CORTEX_E_INVAL;
  if (a->num_seqs == 0 && a->num_tokens != 0) return CORTEX_E_INVAL;
  return CORTEX_OK;
}

template <typename T> int scan_forward_typed(const cortex_scan_t &a, int32_t *status, void *ws, void *stream) {
  if (a.head_dim == 0) {
    switch (a.state_size) {
      case 8: return launch_channel<T, 8>(a, status, ws, stream);
      case 16: return launch_channel<T, 16>(a, status, ws, stream);
      case 32: return launch_channel<T, 32>(a, status, ws, stream);
      default: return launch_channel<T, 64>(a, status, ws, stream);
    }
  }
  switch (a.state_size) {
    case 16: return launch_head<T, 16>(a, status, ws, stream);
    case 32: return launch_head<T, 32>(a, status, ws, stream);
    case 64: return launch_head<T, 64>(a, status, ws, stream);
    default: return launch_head<T, 128>(a, status, ws, stream);
  }
}

template <typename T> int scan_step_typed(const cortex_scan_t &a, int32_t *status, void *stream) {
  if (a.head_dim == 0) {
    switch (a.state_size) {
      case 8: return launch_step<T, 8, false>(a, status, stream);
      case 16: return launch_step<T, 16, false>(a, status, stream);
      case 32: return launch_step<T, 32, false>(a, status, stream);
      default: return launch_step<T, 64, false>(a, status, stream);
    }
  }
  switch (a.state_size) {
    case 16: return launch_step<T, 16, true>(a, status, stream);
    case 32: return launch_step<T, 32, true>(a, status, stream);
    case 64: return launch_step<T, 64, true>(a, status, stream);
    default: return launch_step<T, 128, true>(a, status, stream);
  }
}

}  // namespace cortex

using namespace cortex;

extern "C" size_t cortex_scan_workspace_bytes(int32_t num_tokens, int32_t num_seqs, int32_t channels, int32_t state_size,
                                              int32_t head_dim) {
  if (num_tokens < 0 || num_seqs < 0 || bad_scan_size(channels, 1, state_size, head_dim)) return 0;
  return scratch_bytes(most_slots(num_tokens, num_seqs, channels, state_size, head_dim), channels, state_size);
}

extern "C" int cortex_scan_forward(const cortex_scan_t *args, int32_t *d_status, void *d_ws, size_t ws_bytes, void *stream) {
  const int rc = check_scan(args, false, d_status);
  if (rc != CORTEX_OK) return rc;
  if (args->num_seqs == 0) return CORTEX_OK;
  // Whole sequences per head are a workgroup a unit, and a grid has less than 2^32 threads.
  if (args->head_dim && (int64_t)args->num_seqs * (args->channels / args->head_dim) * ((args->head_dim + 63) / 64) >=
                            (int64_t)1 << 24)
    return CORTEX_E_INVAL;
  if (!d_ws || !aligned16(d_ws)) return CORTEX_E_INVAL;
  const int Q = segment_tokens(args->num_tokens, args->num_seqs, args->channels, args->state_size, args->head_dim);
  const int64_t slots = Q ? chunk_slots(args->num_tokens, args->num_seqs, Q) : 0;
  if (ws_bytes < scratch_bytes(slots, args->channels, args->state_size)) return CORTEX_E_WORKSPACE;
  return args->dtype == CORTEX_BF16 ? scan_forward_typed<bf16_t>(*args, d_status, d_ws, stream)
                                    : scan_forward_typed<float>(*args, d_status, d_ws, stream);
}

extern "C" int cortex_scan_step(const cortex_scan_t *args, int32_t *d_status, void *stream) {
  const int rc = check_scan(args, true, d_status);
  if (rc != CORTEX_OK) return rc;
  if (args->num_seqs == 0) return CORTEX_OK;
  return args->dtype == CORTEX_BF16 ? scan_step_typed<bf16_t>(*args, d_status, stream)
                                    : scan_step_typed<float>(*args, d_status, stream);
}
