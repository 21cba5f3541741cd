// Several new tokens of a sequence at once over the fp16 cache (include/okv_chunk.h): appending with rotation, and attention of the rows, for gfx950.
#include "okv_chunk.h"
#include "okv_host.h"
#include "okv_lanes.h"
#include "okv_report.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "okv.h"

namespace okv {

namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

// ---- the pool -------------------------------------------------------------------------------------

struct Pool {
  _Float16 *kv;
  const int32_t *table, *refused;
  int32_t G, R, gg, st_log2;
  int32_t log2_tiles;                    // tiles of 16 tokens of a block; 30: a contiguous pool, whose sequence is a block
  int32_t width, n_blocks, max_seqs, capacity;
  int64_t block_elems;
};

// Where the K rows of tile t of a sequence begin, for head 0 of the first group; those of other heads are head_offset further, the V rows v_offset behind them
template <int D>
__device__ __forceinline__ int64_t tile_at(const Pool &c, const int32_t *table_row, const int row, const int t) {
  int block = row;
  if (c.table) block = min(max(table_row[t >> c.log2_tiles], 0), c.n_blocks - 1);
  const int tb = t & ((1 << c.log2_tiles) - 1);
  const int64_t slab = (int64_t)2 * c.G * D << (4 + c.st_log2);
  return block * c.block_elems + (tb >> c.st_log2) * slab + (int64_t)(tb & ((1 << c.st_log2) - 1)) * (c.gg * 16 * D);
}
template <int D>
__device__ __forceinline__ int64_t head_offset(const Pool &c, const int g) {
  return (int64_t)(g / c.gg) * (2 * c.gg * D << (4 + c.st_log2)) + g % c.gg * (16 * D);
}
template <int D>
__device__ __forceinline__ int v_offset(const Pool &c) { return c.gg * D << (4 + c.st_log2); }

struct Rows {
  const int32_t *seqs, *starts, *lens;
  int32_t batch, n_rows;
};

// Rows of sequence b: [first, last)
__device__ __forceinline__ void rows_of(const Rows &r, const int b, int &first, int &last) {
  first = min(max(r.starts[b], 0), r.n_rows);
  last = min(max(r.starts[b + 1], first), r.n_rows);
}

// ---- appending ------------------------------------------------------------------------------------

struct Append {
  const _Float16 *k, *v, *q;
  _Float16 *q_out;
  int64_t kv_stride, q_stride, q_out_stride;
  const double *turns;                   // NULL: nothing is turned
  const int32_t *positions;
  int32_t rotated, interleaved, H;
};

__device__ __forceinline__ int sequence_of_row(const Rows &r, const int row) {     // -1: none
  // how many sequences end at or before the row, 64 of them at a time
  const int lane = threadIdx.x & 63;
  int b = 0;
  for (int b0 = 0; b0 < r.batch; b0 += 64) {
    const uint64_t ended = __ballot(b0 + lane < r.batch && r.starts[min(b0 + lane, r.batch - 1) + 1] <= row);
    b += __popcll(ended);
    if (ended != ~0ull) break;
  }
  return b < r.batch && r.starts[b] <= row ? b : -1;
}

constexpr int kAppendWaves = 4;

// A wavefront per row.  A lane has 16 elements of a head, which are eight pairs (or none that turn), and the same ones of every 64 / (D / 16)-th head after it:
// the sines of its pairs are computed once.
template <int D>
__global__ void __launch_bounds__(kAppendWaves * 64) append_kernel(Pool c, Rows r, Append a) {
  const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(blockIdx.x * kAppendWaves + (threadIdx.x >> 6));
  if (row >= r.n_rows) return;
  const int b = __builtin_amdgcn_readfirstlane(sequence_of_row(r, row));
  if (b < 0) return;
  const int s = r.seqs ? r.seqs[b] : b;
  int first, last, len = 0;
  rows_of(r, b, first, last);
  const bool known = s >= 0 && s < c.max_seqs;
  if (known) len = min(max(r.lens[s], 0), c.capacity);
  const int token = len - (last - row);
  constexpr int kUnits = D / 16, kHeads = 64 / kUnits;
  const int unit = lane % kUnits, slot = lane / kUnits, turning = a.rotated / 16;
  const bool turns = a.turns && unit < turning;
  // this lane's two runs of eight elements: x and y of eight pairs, or sixteen in a row
  const bool apart = turns && !a.interleaved;
  const int at0 = apart ? 8 * unit : 16 * unit, at1 = apart ? at0 + a.rotated / 2 : at0 + 8;
  float cosine[8], sine[8];
  if (turns) {
    const double p = a.positions ? a.positions[row] : token;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      double t = p * a.turns[8 * unit + i];
      t -= rint(t);
      sincospif(2.f * (float)t, &sine[i], &cosine[i]);
    }
  }
  auto move = [&](const _Float16 *from, _Float16 *to) {
    half8 x = *reinterpret_cast<const half8 *>(from + at0), y = *reinterpret_cast<const half8 *>(from + at1);
    if (turns) {
      half8 u, w;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = (2 * i) & 7;
        const float e = (float)(!a.interleaved ? x[i] : i < 4 ? x[j] : y[j]), f = (float)(!a.interleaved ? y[i] : i < 4 ? x[j + 1] : y[j + 1]);
        const _Float16 p = (_Float16)(e * cosine[i] - f * sine[i]), q = (_Float16)(e * sine[i] + f * cosine[i]);
        if (!a.interleaved) u[i] = p, w[i] = q;
        else if (i < 4) u[j] = p, u[j + 1] = q;
        else w[j] = p, w[j + 1] = q;
      }
      x = u, y = w;
    }
    *reinterpret_cast<half8 *>(to + at0) = x;
    *reinterpret_cast<half8 *>(to + at1) = y;
  };
  if (a.q)
    for (int h = slot; h < a.H; h += kHeads) move(a.q + row * a.q_stride + h * D, a.q_out + row * a.q_out_stride + h * D);
  if (!known || token < 0 || (c.refused && *c.refused)) return;
  const int64_t at = tile_at<D>(c, c.table + (int64_t)s * c.width, s, token >> 4) + (token & 15) * D;
  for (int g = slot; g < c.G; g += kHeads) {
    _Float16 *to = c.kv + at + head_offset<D>(c, g);
    move(a.k + row * a.kv_stride + g * D, to);
    const _Float16 *v = a.v + row * a.kv_stride + g * D;
    *reinterpret_cast<half8 *>(to + v_offset<D>(c) + 16 * unit) = *reinterpret_cast<const half8 *>(v + 16 * unit);
    *reinterpret_cast<half8 *>(to + v_offset<D>(c) + 16 * unit + 8) = *reinterpret_cast<const half8 *>(v + 16 * unit + 8);
  }
}

// ---- attention ------------------------------------------------------------------------------------

struct Attend {
  const _Float16 *q;
  void *out;
  int64_t q_stride;
  float scale, cap;                      // of scores in units of log 2: scale log2(e), or with a cap scale / cap and cap log2(e)
  int32_t window;                        // 0: none
  const float *slopes;
  const int32_t *prefix;
};

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kRaise = 8.f;            // the maximum is raised when a score is this far above it
// Weights are 2^(s - m + kLift): at most 2^15, and normal numbers in fp16 down to 2^-21 of the largest
constexpr float kLift = 7.f;
constexpr int kKeys = 64;                // of a block
constexpr int kWaves = 4, kTileRows = 32 * kWaves;

// Where 16-byte piece p of row r sits in a block in LDS, in pieces: sixteen rows' same piece, and the four pieces of 32 elements of four rows, are in different banks
template <int D>
__device__ __forceinline__ int piece_at(const int r, const int p) {
  if constexpr (D == 128) return 16 * r + (p ^ (4 * (r & 3) | ((r >> 2) & 3)));
  else return 8 * r + (p ^ (4 * ((r >> 1) & 1) | ((r >> 2) & 3)));
}

__device__ __forceinline__ half8 transposed(const char *lds, const int first, const int second) {
  typedef __attribute__((address_space(3))) short4v *at;
  const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(lds + first)), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(lds + second));
  const half4 x = __builtin_bit_cast(half4, a), y = __builtin_bit_cast(half4, b);
  return half8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// Rows of a workgroup: kTileRows of the n R rows (tokens, and for each its R query heads) of a sequence and KV head.
struct Item {
  int first, n, len, s, tile, g;         // the sequence's first row, its rows, its tokens, its row of the table; s < 0: nothing to do
};
__device__ __forceinline__ Item item_of(const Pool &c, const Rows &r, int piece) {
  const int lane = threadIdx.x & 63;
  Item it;
  it.s = -1;
  for (int b0 = 0; b0 < r.batch; b0 += 64) {
    const int b = b0 + lane;
    int first = 0, last = 0;
    if (b < r.batch) rows_of(r, b, first, last);
    const int tiles = (int)(((int64_t)(last - first) * c.R + kTileRows - 1) / kTileRows);
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int other = __shfl_up(upto, o);
      if (lane >= o) upto += other;
    }
    const int all = __shfl(upto, 63) * c.G;
    if (piece >= all) {
      piece -= all;
      continue;
    }
    const int rank = piece / c.G, at = __popcll(__ballot(upto <= rank));
    it.g = piece % c.G;
    it.tile = __shfl(tiles, at) - 1 - (rank - __shfl(upto - tiles, at));      // the last rows, which see the most keys, first
    it.first = __shfl(first, at), it.n = __shfl(last, at) - it.first;
    const int s = r.seqs ? r.seqs[b0 + at] : b0 + at;
    it.s = s >= 0 && s < c.max_seqs ? s : -2;
    it.len = it.s < 0 ? 0 : min(max(r.lens[s], 0), c.capacity);
    break;
  }
  return it;
}

template <int D, bool WIDE, bool SHAPED>
__global__ void __launch_bounds__(kWaves * 64) chunk_kernel(Pool c, Rows r, Attend a) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * kKeys * D * 2];
  char *const lds_k = lds, *const lds_v = lds + kKeys * D * 2;
  const Item it = item_of(c, r, blockIdx.x);
  if (it.s == -1) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
  const int row = it.tile * kTileRows + wave * 32 + col;                    // of the sequence's n R rows
  const int token = row / c.R, head = it.g * c.R + row % c.R;
  const bool mine = token < it.n;
  const int base = it.len - it.n, pos = base + token;
  const int prefix = a.prefix && it.s >= 0 ? min(max(a.prefix[it.s], 0), it.len) : 0;
  const int from = a.window == 0 || pos < a.window ? 0 : pos - a.window + 1;
  // keys that some row of the tile sees
  const int token0 = it.tile * kTileRows / c.R, token1 = min((it.tile * kTileRows + kTileRows - 1) / c.R, it.n - 1);
  const int pos0 = base + token0, pos1 = base + token1;
  const int from0 = a.window == 0 || pos0 < a.window ? 0 : pos0 - a.window + 1;
  const int end = max(pos1 + 1, prefix);

  half8 qf[D / 16];
  {
    const _Float16 *q = a.q + (it.first + min(token, it.n - 1)) * a.q_stride + head * D + 8 * half;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) qf[k] = *reinterpret_cast<const half8 *>(q + 16 * k);
  }
  const float slope = SHAPED && a.slopes ? a.slopes[head] * kLog2e : 0.f;
  floatx16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = floatx16{};
  float m = -1e30f, l = 0.f;

  const int32_t *table_row = c.table + (int64_t)max(it.s, 0) * c.width;
  const int64_t my_head = head_offset<D>(c, it.g);
  const int behind = v_offset<D>(c);
  const int prefix_blocks = (prefix + kKeys - 1) / kKeys, first_block = from0 / kKeys, last_block = (end + kKeys - 1) / kKeys;
  for (int block = 0; block < last_block; ++block) {
    if (block < first_block && block >= prefix_blocks) {
      block = first_block - 1;
      continue;
    }
    const int key0 = block * kKeys;
    __syncthreads();
    constexpr int kPieces = D / 8;
#pragma unroll
    for (int i = 0; i < kKeys * kPieces / (kWaves * 64); ++i) {
      const int u = i * kWaves * 64 + threadIdx.x, key = u / kPieces, piece = u % kPieces;
      const int t = min((key0 + key) >> 4, (it.len - 1) >> 4);
      const _Float16 *k = c.kv + tile_at<D>(c, table_row, it.s, t) + my_head + (key & 15) * D + 8 * piece;
      *reinterpret_cast<u32x4 *>(lds_k + 16 * piece_at<D>(key, piece)) = *reinterpret_cast<const u32x4 *>(k);
      *reinterpret_cast<u32x4 *>(lds_v + 16 * piece_at<D>(key, piece)) = *reinterpret_cast<const u32x4 *>(k + behind);
    }
    __syncthreads();
    // scores: keys 32 b + 8 (i / 4) + 4 half + i % 4 of this lane's row
    floatx16 x[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      x[b] = floatx16{};
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const half8 kf = *reinterpret_cast<const half8 *>(lds_k + 16 * piece_at<D>(32 * b + col, 2 * k + half));
        x[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[k], x[b], 0, 0, 0);
      }
    }
    const bool whole = (key0 + kKeys - 1 <= pos0 && key0 >= (a.window == 0 || pos1 < a.window ? 0 : pos1 - a.window + 1)) || key0 + kKeys <= prefix;
    float top = -INFINITY;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + 32 * b + 8 * (i / 4) + 4 * half + i % 4;
        float s = x[b][i] * a.scale;
        if constexpr (SHAPED) {
          if (a.cap != 0.f) s = a.cap * tanhf(s);
          s = fmaf(-slope, (float)abs(pos - key), s);
        }
        if (!whole && !((key <= pos && key >= from) || key < prefix)) s = -INFINITY;
        x[b][i] = s;
        top = fmaxf(top, s);
      }
    top = max_with_lane_xor<32>(top);
    if (__ballot(top > m + kRaise)) {
      const float to = top > m + kRaise ? top : m, by = __builtin_amdgcn_exp2f(m - to);
      l *= by;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] *= by;
      m = to;
    }
    half8 hi[4], lo[4];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(x[b][i] - m + kLift);
        l += p;
        hi[2 * b + i / 8][i % 8] = (_Float16)p;
        if constexpr (WIDE) lo[2 * b + i / 8][i % 8] = (_Float16)(p - (float)(_Float16)p);
      }
    // results: elements 32 e + 8 (i / 4) + 4 half + i % 4 of this lane's row
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int key = 16 * t + 4 * half + (lane & 15) / 4, piece = 4 * e + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        half8 vf = transposed(lds_v, 16 * piece_at<D>(key, piece) + 8 * (lane & 1), 16 * piece_at<D>(key + 8, piece) + 8 * (lane & 1));
        if (!whole) {
          // numbers that are not finite may be of keys that a row does not see, and 0 times them is not 0: they go in apart, by whether a row sees them
          half8 above, below, rest;
          bool odd = false;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float v = (float)vf[j];
            const bool fine = fabsf(v) < INFINITY;
            above[j] = fine || v < 0.f ? (_Float16)0.f : (_Float16)1.f;
            below[j] = fine || v > 0.f ? (_Float16)0.f : (_Float16)1.f;
            rest[j] = fine ? vf[j] : (_Float16)0.f;
            odd |= !fine;
          }
          vf = rest;
          if (__ballot(odd)) {
            const floatx16 up = __builtin_amdgcn_mfma_f32_32x32x16_f16(above, hi[t], floatx16{}, 0, 0, 0);
            const floatx16 down = __builtin_amdgcn_mfma_f32_32x32x16_f16(below, hi[t], floatx16{}, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[e][i] += (up[i] != 0.f ? INFINITY : 0.f) - (down[i] != 0.f ? INFINITY : 0.f);
          }
        }
        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, hi[t], o[e], 0, 0, 0);
        if constexpr (WIDE) o[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, lo[t], o[e], 0, 0, 0);
      }
  }
  if (!mine) return;
  l = sum_with_lane_xor<32>(l);
  const float over = l == 0.f ? 0.f : 1.f / l;
  const int64_t to = ((int64_t)(it.first + token) * (c.G * c.R) + head) * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      floatx4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = o[e][4 * i + j] * over;
      const int64_t at = to + 32 * e + 8 * i + 4 * half;
      if constexpr (WIDE) *reinterpret_cast<floatx4 *>(static_cast<float *>(a.out) + at) = y;
      else *reinterpret_cast<half4 *>(static_cast<_Float16 *>(a.out) + at) = half4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
    }
}

// ---- host -------------------------------------------------------------------------------------------

bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

const char *shape_problem(const okv_layer_pool *c) {
  if (!c) return "the pool is NULL";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 16)
    return "n_kv_heads must be in [1, 1024] and n_q_heads 1 to 16 times that";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->max_seqs < 1) return "max_seqs must be at least 1";
  if (c->block_tokens == 0) {
    if (c->max_ctx < 16 || c->max_ctx % 16 || c->max_ctx > 0x3fffffff) return "contiguous pools need max_ctx >= 16, a multiple of 16 and below 2^30";
    return nullptr;
  }
  if (c->block_tokens < 16 || c->block_tokens > 1024 || (c->block_tokens & (c->block_tokens - 1))) return "block_tokens must be 0 or a power of two in [16, 1024]";
  if (c->max_blocks_per_seq < 1 || (int64_t)c->max_blocks_per_seq * c->block_tokens > 0x3fffffff) return "a sequence's capacity must be in [1, 2^30) tokens";
  if (c->n_blocks < 1 || c->n_blocks > 0x7fffffff) return "n_blocks must be in [1, 2^31)";
  return nullptr;
}
const char *problem(const okv_layer_pool *c, const okv_rows *r) {
  if (const char *why = shape_problem(c)) return why;
  if (!c->pool || (c->block_tokens && !c->block_table)) return "NULL pointer";
  if (!aligned(c->pool, 16)) return "the pool is not 16-byte aligned";
  if (!r) return "the rows are NULL";
  if (r->batch < 0 || r->batch > OKV_CHUNK_MAX_BATCH || r->n_rows < 0) return "batch must be in [0, 4096] and n_rows not negative";
  if (r->batch && (!r->starts || !r->lens)) return "NULL pointer";
  if (!r->seqs && r->batch > c->max_seqs) return "more sequences than the table has rows";
  return nullptr;
}
Pool pool_of(const okv_layer_pool *c) {
  const bool paged = c->block_tokens != 0;
  const int32_t slice = paged ? c->block_tokens : c->max_ctx;
  Pool p;
  p.kv = static_cast<_Float16 *>(c->pool);
  p.table = paged ? c->block_table : nullptr, p.refused = c->refused;
  p.G = c->n_kv_heads, p.R = c->n_q_heads / c->n_kv_heads;
  p.gg = kv_head_group(p.G, c->head_dim), p.st_log2 = slab_tiles_log2(p.G, c->head_dim, slice);
  p.log2_tiles = paged ? 31 - __builtin_clz((unsigned)c->block_tokens / 16) : 30;
  p.width = paged ? c->max_blocks_per_seq : 1, p.n_blocks = paged ? (int32_t)c->n_blocks : c->max_seqs, p.max_seqs = c->max_seqs;
  p.capacity = paged ? c->max_blocks_per_seq * c->block_tokens : c->max_ctx;
  p.block_elems = (int64_t)2 * p.G * c->head_dim * slice;
  return p;
}
int hip_result(const char *who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OKV_OK : report(OKV_EHIP, "%s: %s", who, hipGetErrorString(e));
}

}  // namespace

}  // namespace okv

using namespace okv;

extern "C" {

int okv_rope_append(const okv_layer_pool *c, const okv_rows *r, const okv_rope *rope, const void *k, const void *v, int64_t kv_stride, const void *q,
                    int64_t q_stride, void *q_out, int64_t q_out_stride, void *stream) {
  const char *const who = "okv_rope_append";
  if (const char *why = problem(c, r)) return report(OKV_EINVAL, "%s: %s", who, why);
  const int32_t d = c->head_dim;
  if (rope && (rope->rotated < 0 || rope->rotated > d || rope->rotated % 16)) return report(OKV_EINVAL, "%s: rotated must be a multiple of 16 in [0, head_dim]", who);
  if (rope && rope->rotated && !rope->turns) return report(OKV_EINVAL, "%s: NULL pointer", who);
  if (kv_stride < (int64_t)c->n_kv_heads * d || kv_stride % 8) return report(OKV_EINVAL, "%s: kv_stride must be a multiple of 8 and at least n_kv_heads * head_dim", who);
  if ((q == nullptr) != (q_out == nullptr)) return report(OKV_EINVAL, "%s: q and q_out come together", who);
  for (const int64_t s : {q_stride, q_out_stride})
    if (q && (s < (int64_t)c->n_q_heads * d || s % 8)) return report(OKV_EINVAL, "%s: q_stride and q_out_stride must be multiples of 8 and at least n_q_heads * head_dim", who);
  if (q && q == q_out && q_stride != q_out_stride) return report(OKV_EINVAL, "%s: queries that are turned in place keep their stride", who);
  if (r->batch == 0 || r->n_rows == 0) return OKV_OK;
  if (!k || !v) return report(OKV_EINVAL, "%s: NULL pointer", who);
  for (const void *p : {k, v, q, static_cast<const void *>(q_out)})
    if (!aligned(p, 16)) return report(OKV_EINVAL, "%s: pointer not 16-byte aligned", who);
  const Pool pool = pool_of(c);
  const Rows rows{r->seqs, r->starts, r->lens, r->batch, r->n_rows};
  Append a;
  a.k = static_cast<const _Float16 *>(k), a.v = static_cast<const _Float16 *>(v), a.q = static_cast<const _Float16 *>(q), a.q_out = static_cast<_Float16 *>(q_out);
  a.kv_stride = kv_stride, a.q_stride = q_stride, a.q_out_stride = q_out_stride;
  const bool turns = rope && rope->rotated;
  a.turns = turns ? rope->turns : nullptr, a.positions = turns ? rope->positions : nullptr;
  a.rotated = turns ? rope->rotated : 0, a.interleaved = turns && rope->interleaved, a.H = c->n_q_heads;
  const dim3 grid((unsigned)((r->n_rows + (int64_t)kAppendWaves - 1) / kAppendWaves)), block(kAppendWaves * 64);
  if (d == 128) hipLaunchKernelGGL(append_kernel<128>, grid, block, 0, static_cast<hipStream_t>(stream), pool, rows, a);
  else hipLaunchKernelGGL(append_kernel<64>, grid, block, 0, static_cast<hipStream_t>(stream), pool, rows, a);
  return hip_result(who);
}

int64_t okv_chunk_workspace_bytes(const okv_layer_pool *c) {
  if (const char *why = shape_problem(c)) return report(OKV_EINVAL, "okv_chunk_workspace_bytes: %s", why);
  return 0;
}

int okv_chunk_attn(const okv_layer_pool *c, const okv_rows *r, const okv_chunk *a, const void *q, int64_t q_stride, void *out, void *stream) {
  const char *const who = "okv_chunk_attn";
  if (const char *why = problem(c, r)) return report(OKV_EINVAL, "%s: %s", who, why);
  if (!a) return report(OKV_EINVAL, "%s: NULL pointer", who);
  if (!(a->scale >= 0.f && a->scale < INFINITY) || !(a->cap >= 0.f && a->cap < INFINITY)) return report(OKV_EINVAL, "%s: scale and cap must be finite and not negative", who);
  if (a->window < 0) return report(OKV_EINVAL, "%s: window must not be negative", who);
  if (a->out_dtype != 0 && a->out_dtype != 1) return report(OKV_EINVAL, "%s: out_dtype must be 0 or 1", who);
  const int32_t d = c->head_dim;
  if (q_stride < (int64_t)c->n_q_heads * d || q_stride % 8) return report(OKV_EINVAL, "%s: q_stride must be a multiple of 8 and at least n_q_heads * head_dim", who);
  if (r->batch == 0 || r->n_rows == 0) return OKV_OK;
  if (!q || !out) return report(OKV_EINVAL, "%s: NULL pointer", who);
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(a->slopes, 4) || !aligned(a->prefix, 4)) return report(OKV_EINVAL, "%s: q and out must be 16-byte aligned, slopes and prefix 4", who);
  const int64_t need = okv_chunk_workspace_bytes(c);
  if (need && (!a->workspace || a->workspace_bytes < need || !aligned(a->workspace, 256)))
    return report(OKV_ENOSPC, "%s: the workspace must be %lld bytes, 256-byte aligned", who, (long long)need);
  const Pool pool = pool_of(c);
  const Rows rows{r->seqs, r->starts, r->lens, r->batch, r->n_rows};
  // a tile of rows begins at a sequence's first row
  const int64_t tiles = ((int64_t)r->n_rows * pool.R + kTileRows - 1) / kTileRows + std::min(r->batch, r->n_rows), pieces = tiles * pool.G;
  if (pieces > 0x7fffffff / 256) return report(OKV_EINVAL, "%s: too many rows for a call", who);
  Attend x;
  x.q = static_cast<const _Float16 *>(q), x.out = out, x.q_stride = q_stride;
  const float scale = a->scale != 0.f ? a->scale : 1.f / sqrtf((float)d);
  x.scale = a->cap != 0.f ? scale / a->cap : scale * kLog2e, x.cap = a->cap * kLog2e;
  x.window = a->window, x.slopes = a->slopes, x.prefix = a->prefix;
  const bool wide = a->out_dtype == 1, shaped = a->cap != 0.f || a->slopes;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)pieces), dim3(kWaves * 64), 0, static_cast<hipStream_t>(stream), pool, rows, x); };
  auto typed = [&](auto d_) {
    constexpr int D = decltype(d_)::value;
    if (wide) shaped ? launch(chunk_kernel<D, true, true>) : launch(chunk_kernel<D, true, false>);
    else shaped ? launch(chunk_kernel<D, false, true>) : launch(chunk_kernel<D, false, false>);
  };
  if (d == 128) typed(std::integral_constant<int, 128>{});
  else typed(std::integral_constant<int, 64>{});
  return hip_result(who);
}

}  // extern "C"
