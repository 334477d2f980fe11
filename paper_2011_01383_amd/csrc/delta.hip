// The gated delta rule, for prompts and for single tokens.
//
//   S <- a S,  u = beta (v - S k),  S <- S + u k^T,  y = scale S q
//
// Rows of a head's state (one per value channel) share nothing but k, q, a and
// beta.  Eight lanes hold a row, four entries of each 32 a lane, so that a row's
// loads and stores are whole 128-byte pieces; a wave holds sixteen rows.  The states' bytes bound it:
// 64 rows of 32 heads of 128 by 128 are 268 MB, 46 us (5.8 TB/s: some stay in the last-level cache), one row 5 us.
#include "delta_chunk.hpp"

namespace cortex {

constexpr int kDeltaWaves = 4;           // tiles of 16 rows in a workgroup, of neighbouring number
constexpr int kDeltaTile = 16;

// Sum over the eight lanes that share a row.
__device__ __forceinline__ float row_sum(float v) {
  v += shifted<0xb1>(v, 0.0f);           // quad_perm: the neighbour
  v += shifted<0x4e>(v, 0.0f);           // the other pair of four
  v += shifted<0x141>(v, 0.0f);          // the other four of eight
  return v;
}

// Four consecutive elements.
template <typename T, bool WIDE> __device__ __forceinline__ void load4(const T *p, float (&v)[4]) {
  if constexpr (WIDE) Pack<T, 4>::load(p, v);
  else
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_float<T>(p[i]);
}

template <typename T, int K, bool WIDE>
__global__ void __launch_bounds__(64 * kDeltaWaves) delta_step_kernel(cortex_delta_t p, int32_t *status, int64_t units) {
  constexpr int C = K / 32;
  if (entry_status(status) != 0) return;
  const int lane = (int)threadIdx.x & 63, part = lane & 7, row8 = lane >> 3;
  const int64_t unit = (int64_t)blockIdx.x * kDeltaWaves + (threadIdx.x >> 6);
  if (unit >= units) return;
  const int V = p.value_dim, tiles = V / kDeltaTile, per = p.heads * tiles;
  const int seq = (int)(unit / per), rest = (int)(unit % per), head = rest / tiles;
  const int v0 = rest % tiles * kDeltaTile + row8, g = head / (p.heads / p.key_heads);
  int pool = -1;
  if (p.state_in || p.state_out) {
    pool = state_row(p.state_index, seq, p.state_rows, status);
    if (pool < -1) return;
  }
  const int64_t at = (((int64_t)pool * p.heads + head) * V + v0) * K + part * 4;
  typedef float vec __attribute__((ext_vector_type(4)));
  vec h[2][C];
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c)
      h[r][c] = p.state_in && pool >= 0 ? *(const vec *)(p.state_in + at + r * 8 * K + c * 32) : vec{0.0f, 0.0f, 0.0f, 0.0f};
  const T *qs = (const T *)p.q + g * K + part * 4, *ks = (const T *)p.k + g * K + part * 4;
  const T *vs = (const T *)p.v + (int64_t)head * V + v0;
  T *ys = (T *)p.y + (int64_t)head * V + v0;
  const int64_t t = seq;
  float q[C][4], k[C][4], v[2];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load4<T, WIDE>(qs + t * p.q_ld + c * 32, q[c]);
    load4<T, WIDE>(ks + t * p.k_ld + c * 32, k[c]);
  }
  v[0] = to_float<T>(vs[t * p.v_ld]);
  v[1] = to_float<T>(vs[t * p.v_ld + 8]);
  float a = 1.0f;
  if (p.A) {
    const float raw = to_float<T>(((const T *)p.dt)[t * p.dt_ld + head]) + (p.dt_bias ? p.dt_bias[head] : 0.0f);
    a = fast_exp2((p.softplus ? softplus(raw) : raw) * decay_rate(p.A[head]));
  }
  const float b = to_float<T>(((const T *)p.b)[t * p.b_ld + head]), beta = p.sigmoid ? sigmoid(b) : b;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    float dot = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[r][c][i] *= a;
        dot = __builtin_fmaf(h[r][c][i], k[c][i], dot);
      }
    const float u = beta * (v[r] - row_sum(dot));
    float y = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[r][c][i] = __builtin_fmaf(u, k[c][i], h[r][c][i]);
        y = __builtin_fmaf(h[r][c][i], q[c][i], y);
      }
    y = row_sum(y) * p.scale;
    if (part == 0) ys[t * p.y_ld + r * 8] = from_float<T>(y);
    if (p.state_out && pool >= 0)
#pragma unroll
      for (int c = 0; c < C; ++c) *(vec *)(p.state_out + at + r * 8 * K + c * 32) = h[r][c];
  }
}

static bool launched() { return hipGetLastError() == hipSuccess; }

template <typename T, int K> int launch_step_of(const cortex_delta_t &a, int32_t *status, void *stream) {
  const int64_t units = (int64_t)a.num_seqs * a.heads * (a.value_dim / kDeltaTile);
  const unsigned grid = (unsigned)((units + kDeltaWaves - 1) / kDeltaWaves);
  constexpr uintptr_t mask = 4 * sizeof(T) - 1;
  const bool wide = a.q_ld % 4 == 0 && a.k_ld % 4 == 0 && ((uintptr_t)a.q & mask) == 0 && ((uintptr_t)a.k & mask) == 0;
  if (wide) delta_step_kernel<T, K, true><<<grid, 64 * kDeltaWaves, 0, (hipStream_t)stream>>>(a, status, units);
  else delta_step_kernel<T, K, false><<<grid, 64 * kDeltaWaves, 0, (hipStream_t)stream>>>(a, status, units);
  return launched() ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T, int K, bool WIDE>
void launch_walk(const cortex_delta_t &a, int32_t *status, const ChunkMap *maps, hipStream_t st) {
  constexpr int kColumns = 16 * kChunkWaves;
  const int64_t units = (int64_t)a.num_seqs * a.heads * ((a.value_dim + kColumns - 1) / kColumns);
  chunk_walk_kernel<T, K, WIDE><<<(unsigned)units, kChunkThreads, 0, st>>>(a, status, maps);
}

// Workgroups that a launch of segments may have, and so the rows of 16 that they leave.
constexpr int64_t kMaxSegmentTiles = 2048;

// Tokens of a segment, 0 for whole sequences.  By the time of a chunk in one launch of
// workgroups (one a CU): 2 us with outputs, 1.5 without, 1.5 for joining two segments and 12 for the two
// launches more.  The host knows no lengths: sequences are taken as equally long, of one token at least.  24,576 tokens of one head
// of 128 by 128 take 156 us in segments and 650 whole, 8,192 tokens of 2 heads 99 and 227, of 8
// heads 197 and 238, 2,048 tokens of 4 heads of 64 by 64 38 and 58.
static int segment_tokens(int64_t T, int64_t S, int64_t heads, int64_t K, int64_t V) {
  const int64_t columns = heads * V / 16, maps = heads * (V + K) / 16;
  auto rounds = [](int64_t workgroups) { return (double)((workgroups + 255) / 256); };
  const int64_t length = T > S ? (T + S - 1) / S : 1;
  double best = 0.8 * 2.0 * rounds(S * columns) * (double)((length + kChunk - 1) / kChunk);
  int Q = 0;
  for (int64_t chunks = 4; chunks <= 512; chunks *= 2) {
    if (chunk_slots(T, S, (int)chunks * kChunk) * maps > kMaxSegmentTiles) continue;
    const int64_t each = (length + chunks * kChunk - 1) / (chunks * kChunk), segments = S * each;
    if (each < 2) break;                         // nothing is cut
    const double time = (double)chunks * (1.5 * rounds((segments - S) * maps) + 2.0 * rounds(segments * columns)) + 1.5 * (double)each + 12.0;
    if (time < best) {
      best = time;
      Q = (int)chunks * kChunk;
    }
  }
  return Q;
}

// The workspace: what the first launch leaves for every chunk and head, the segments' states, and a line that is
// written and never read.
static size_t map_bytes(int64_t T, int64_t S, int64_t heads) { return (size_t)(chunk_slots(T, S, kChunk) * heads) * sizeof(ChunkMap); }
static size_t segment_bytes(int64_t K) { return (size_t)(kMaxSegmentTiles * 16 * K) * sizeof(float) + 256; }

// Eight waves to 16 columns while there are fewer than four workgroups of them a CU, else a wave each: at 512
// units 290 us against 462 (8,192 tokens of 2 prompts, 32 heads of 128 by 128), at 768 202 against 258 (12,000 tokens
// of 6, 16 heads of 64 by 128), at 1,024 300 against 314 (8,192 of 4) and 46 against 35 (4,096 of 32, 8 heads of
// 64 by 64), at 2,048 323 against 225 (8,192 of 8).
static bool few_columns(int64_t S, int64_t heads, int64_t V) { return S * heads * (V / 16) < 1024; }

template <typename T, int K, bool WIDE> int launch_chunks_of(const cortex_delta_t &a, int32_t *status, ChunkMap *maps, void *stream) {
  const hipStream_t st = (hipStream_t)stream;
  const int64_t chunks = chunk_slots(a.num_tokens, a.num_seqs, kChunk) * a.heads;
  const int64_t units = (int64_t)a.num_seqs * a.heads * (a.value_dim / 16);
  const bool few = few_columns(a.num_seqs, a.heads, a.value_dim);
  if (few) chunk_maps_kernel<T, K, false, WIDE><<<blocks_of_units(chunks), kChunkThreads, 0, st>>>(a, status, maps, chunks);
  else chunk_maps_kernel<T, K, true, WIDE><<<blocks_of_units(chunks), kChunkThreads, 0, st>>>(a, status, maps, chunks);
  if (!launched()) return CORTEX_E_HIP;
  if (!few) {
    launch_walk<T, K, WIDE>(a, status, maps, st);
    return launched() ? CORTEX_OK : CORTEX_E_HIP;
  }
  const int Q = segment_tokens(a.num_tokens, a.num_seqs, a.heads, K, a.value_dim);
  float *segments = (float *)((char *)maps + map_bytes(a.num_tokens, a.num_seqs, a.heads));
  float *nowhere = segments + kMaxSegmentTiles * 16 * K;
  if (!Q) {
    chunk_chain_kernel<T, K, 0, WIDE><<<(unsigned)units, kChainThreads, 0, st>>>(a, status, maps, segments, nowhere, 0);
    return launched() ? CORTEX_OK : CORTEX_E_HIP;
  }
  const int64_t slots = chunk_slots(a.num_tokens, a.num_seqs, Q) * a.heads;
  const int64_t tiles = slots * ((a.value_dim + K) / 16), columns = slots * (a.value_dim / 16);
  chunk_chain_kernel<T, K, 1, WIDE><<<(unsigned)tiles, kChainThreads, 0, st>>>(a, status, maps, segments, nowhere, Q);
  if (!launched()) return CORTEX_E_HIP;
  enter_segments_kernel<K><<<(unsigned)units, kChunkThreads, 0, st>>>(a, status, segments, Q);
  if (!launched()) return CORTEX_E_HIP;
  chunk_chain_kernel<T, K, 2, WIDE><<<(unsigned)columns, kChainThreads, 0, st>>>(a, status, maps, segments, nowhere, Q);
  return launched() ? CORTEX_OK : CORTEX_E_HIP;
}

template <typename T, int K> int launch_chunks(const cortex_delta_t &a, int32_t *status, ChunkMap *maps, void *stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool wide = a.q_ld % V == 0 && a.k_ld % V == 0 && aligned16(a.q) && aligned16(a.k);
  return wide ? launch_chunks_of<T, K, true>(a, status, maps, stream) : launch_chunks_of<T, K, false>(a, status, maps, stream);
}

template <typename T> int launch_forward(const cortex_delta_t &a, int32_t *status, void *ws, void *stream) {
  switch (a.key_dim) {
    case 32: return launch_chunks<T, 32>(a, status, (ChunkMap *)ws, stream);
    case 64: return launch_chunks<T, 64>(a, status, (ChunkMap *)ws, stream);
    default: return launch_chunks<T, 128>(a, status, (ChunkMap *)ws, stream);
  }
}

template <typename T> int launch_step(const cortex_delta_t &a, int32_t *status, void *stream) {
  switch (a.key_dim) {
    case 32: return launch_step_of<T, 32>(a, status, stream);
    case 64: return launch_step_of<T, 64>(a, status, stream);
    default: return launch_step_of<T, 128>(a, status, stream);
  }
}

static bool bad_delta_size(int32_t heads, int32_t key_heads, int32_t K, int32_t V) {
  if (heads < 1 || key_heads < 1 || heads % key_heads) return true;
  if (V < 16 || V > 256 || V % 16 || (int64_t)heads * V > kMaxChannels) return true;
  return K != 32 && K != 64 && K != 128;
}

static int check_delta(const cortex_delta_t *a, bool step, int32_t *status) {
  if (!a || !status) return CORTEX_E_INVAL;
  if (bad_delta_size(a->heads, a->key_heads, a->key_dim, a->value_dim)) return CORTEX_E_INVAL;
  if (bad_batch(a->dtype, a->num_seqs, a->num_tokens, a->heads * a->value_dim, a->state_rows, a->state_index,
                a->state_in || a->state_out))
    return CORTEX_E_INVAL;
  if (step ? a->num_tokens != a->num_seqs : !a->seq_offsets) return CORTEX_E_INVAL;
  const int64_t qk = (int64_t)a->key_heads * a->key_dim, vy = (int64_t)a->heads * a->value_dim;
  if (a->q_ld < qk || a->k_ld < qk || a->v_ld < vy || a->y_ld < vy || a->b_ld < a->heads || (a->A && a->dt_ld < a->heads))
    return CORTEX_E_INVAL;
  if (a->q_ld > kMaxRowStride || a->k_ld > kMaxRowStride || a->v_ld > kMaxRowStride || a->y_ld > kMaxRowStride ||
      a->b_ld > kMaxRowStride || (a->A && a->dt_ld > kMaxRowStride))
    return CORTEX_E_INVAL;
  if (!aligned16(a->state_in) || !aligned16(a->state_out)) return CORTEX_E_INVAL;
  if (a->num_tokens > 0 && (!a->q || !a->k || !a->v || !a->b || !a->y || (a->A && !a->dt))) return CORTEX_E_INVAL;
  if (a->num_seqs == 0 && a->num_tokens != 0) return CORTEX_E_INVAL;
  // A unit is a wave, four of them a workgroup, and a grid has less than 2^32 threads.
  if ((int64_t)a->num_seqs * a->heads * (a->value_dim / kDeltaTile) >= (int64_t)1 << 25) return CORTEX_E_INVAL;
  return CORTEX_OK;
}

}  // namespace cortex

using namespace cortex;

extern "C" size_t cortex_delta_workspace_bytes(int32_t num_tokens, int32_t num_seqs, int32_t heads, int32_t key_dim,
                                               int32_t value_dim) {
  if (num_tokens < 0 || num_seqs < 0 || bad_delta_size(heads, 1, key_dim, value_dim)) return 0;
  return map_bytes(num_tokens, num_seqs, heads) + segment_bytes(key_dim);
}

extern "C" int32_t cortex_delta_segment_tokens(int32_t num_tokens, int32_t num_seqs, int32_t heads, int32_t key_dim, int32_t value_dim) {
  if (num_tokens < 0 || num_seqs < 1 || bad_delta_size(heads, 1, key_dim, value_dim)) return 0;
  return few_columns(num_seqs, heads, value_dim) ? segment_tokens(num_tokens, num_seqs, heads, key_dim, value_dim) : 0;
}

extern "C" int cortex_delta_forward(const cortex_delta_t *args, int32_t *d_status, void *d_ws, size_t ws_bytes, void *stream) {
  const int rc = check_delta(args, false, d_status);
  if (rc != CORTEX_OK) return rc;
  if (args->num_seqs == 0) return CORTEX_OK;
  // a workgroup a chunk and head, and a grid has less than 2^32 threads
  if (chunk_slots(args->num_tokens, args->num_seqs, kChunk) * args->heads > (int64_t)1 << 23) return CORTEX_E_INVAL;
  if (!d_ws || !aligned16(d_ws)) return CORTEX_E_INVAL;
  if (ws_bytes < map_bytes(args->num_tokens, args->num_seqs, args->heads) + segment_bytes(args->key_dim)) return CORTEX_E_WORKSPACE;
  return args->dtype == CORTEX_BF16 ? launch_forward<bf16_t>(*args, d_status, d_ws, stream)
                                    : launch_forward<float>(*args, d_status, d_ws, stream);
}

extern "C" int cortex_delta_step(const cortex_delta_t *args, int32_t *d_status, void *stream) {
  const int rc = check_delta(args, true, d_status);
  if (rc != CORTEX_OK) return rc;
  if (args->num_seqs == 0) return CORTEX_OK;
  return args->dtype == CORTEX_BF16 ? launch_step<bf16_t>(*args, d_status, stream)
                                    : launch_step<float>(*args, d_status, stream);
}
