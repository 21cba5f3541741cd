// A paged KV cache held in 8 bits (include/okv_cache8.h): storing, reading back, and decode attention, for gfx950.
//
// Decode attention out[h] = sum_i softmax_i(q_h . k_i / sqrt(d)) v_i reads every key and value once: bound by HBM, 2 d bytes per key
// and KV head here, half of an fp16 cache's.  The work on a byte is therefore twice the fp16 kernel's, and is kept small:
//
//   * a tile of 32 keys is stored in the order in which lanes feed it to 16x16x32 matrix-core instructions.  A lane's 16 bytes are the
//     operands of two of them, so nothing is transposed or moved between lanes: scores are K (rows: keys) times q (columns: the
//     query heads of the KV head), and the result's layout -- lane l has keys 4 (l / 16) + 0..3 of query l % 16, twice -- is,
//     with V's keys stored in that order, the operand layout of the second product, V^T (rows: elements) times the weights;
//   * codes become fp16 numbers exactly (int8: a byte shuffle that makes 1024 + u, and a subtraction; e4m3: the conversion instruction), the
//     scale of K multiplies the scores in fp32, that of V goes into the weights' exponent;
//   * weights go into the second product as two fp16 numbers, hi and lo, whose products are added up apart: each is off by 2^-22 of itself or by 2^-42 of
//     the largest, whichever is more (see Softmax8).  One rounded to 11 bits would leave errors of 1e-4 of the result, which an fp32 output
//     would show;
//   * only whole tiles are in codes, so the loop over them has no masks; the up to 32 keys in a sequence's fp16 tail are attended
//     by wavefronts of their own in the same launch, which also store the appended row and quantise a tail that is full.
//
// The keys of a launch are cut into equal stretches of tiles over the sequences laid end to end, a wavefront per (stretch, KV head);
// partial results (max, sum, weighted sum) are joined by a second launch (short sequences are not cut and need none).  A step whose layers'
// inputs are all there attends up to 32 layers in one launch, the stretches that much longer.
//
// Measured, us a launch: attention over 810 MB (4 layers of 32 x 768 keys x 32 heads, d = 128) 132 (6.1 TB/s), 159 where every tail is full and is
// quantised; over 1.20 GB (2 layers of 128 x 512..4096 keys, 8 KV heads of 4) 184 (6.5 TB/s), its plan 5, joining 5.6; over 713 MB (2 layers of 2
// documents of up to 131072 keys) 115 (6.2 TB/s), joining 6.  Storing 24 prompts of 100..2000 x 32 heads x 4 layers 500 (2.44 GB, 4.9 TB/s:
// bound by HBM), reading them back 443 (5.5 TB/s).  What is counted as read past L2 is within 1 % of the bytes of codes, scales and tails.
#include "okv_cache8.h"
#include "okv_host.h"
#include "okv_lanes.h"
#include "okv_report.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "okv.h"

namespace okv {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = OKV8_TILE;
// Wavefronts of the part of a launch that reads codes: one per SIMD at d = 128, with 8 KiB in flight each, two at d = 64, where a tile is half that.  us of a
// case of 4 layers x 2 of 32 x 1500 keys x 32 heads (d = 64) with 1024 / 2048 / 4096 of them 367 / 250 / 252; at d = 128 with 1024 / 1536 /
// 2048: 32 x 768 keys x 32 heads 281 / 288 / 280, ragged grouped heads 381 / 399 / 396, two long documents 236 / 235 / 234.
constexpr int kWaves = 1024;
constexpr int kMinSpan = 2;              // tiles of a stretch at least

struct Shape8 {
  int32_t G, R, gg, log2_T, max_seqs, max_pages, n_pages;
};

struct Cache8 {
  uint8_t *codes;          // of the (first) layer
  float *scales;
  _Float16 *tails;
  const int32_t *table, *refused;
  Shape8 s;
};
// Whether nothing may be written: the pages for it could not be taken, and the last token is not the new one
__device__ __forceinline__ bool refused(const Cache8 &c) { return c.refused && *c.refused; }

// ---- codes ------------------------------------------------------------------------------------------

// 4 codes -> 4 fp16 numbers
template <int FMT>
__device__ __forceinline__ void unpack4(const uint32_t w, half2v &a, half2v &b) {
  if constexpr (FMT == OKV8_INT8) {
    const half2v bias = {(_Float16)1152.f, (_Float16)1152.f};
    a = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - bias;
    b = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - bias;
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
  }
}
template <int FMT>
__device__ __forceinline__ half8 unpack8(const uint32_t w0, const uint32_t w1) {
  half2v a, b, c, d;
  unpack4<FMT>(w0, a, b);
  unpack4<FMT>(w1, c, d);
  return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float largest_of(const half8 x) {      // of the magnitudes' bits, as a number: infinities and NaN are the largest
  const u32x4 w = __builtin_bit_cast(u32x4, x);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  return (float)m;
}

// The scale for numbers whose largest magnitude has these bits (see okv_cache8.h)
template <int FMT>
__device__ __forceinline__ float scale_of(const float bits) {
  const uint32_t b = (uint32_t)bits;
  if (b >= 0x7c00u) return __builtin_nanf("");
  const float a = (float)__builtin_bit_cast(_Float16, (uint16_t)b);
  const float s = a * (FMT == OKV8_INT8 ? 1.f / 127.f : 1.f / 448.f);
  return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) + 4095u) & ~4095u);
}

// x / scale and its rounding.  A product with the reciprocal (1 unit in the last place off) and one correction by the exact remainder: a quotient
// that lies on a rounding boundary comes out exactly, any other on its side, because it is 2^-21 away from it (okv_cache8.h).  Whole
// numbers are rounded by an addition: 1.5 2^23 + 128 + y has the code in its last byte.
template <int FMT>
__device__ __forceinline__ u32x2 quantise8(const half8 x, const float scale) {
  const bool some = scale > 0.f;                     // scale 0 or NaN: codes 0
  const float over = some ? __builtin_amdgcn_rcpf(scale) : 0.f, by = some ? scale : 0.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = (float)x[i], q = v * over;
    y[i] = fmaf(fmaf(-q, by, v), over, q);
  }
  if (!some)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = 0.f;
  u32x2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w = 0;
    if constexpr (FMT == OKV8_INT8) {
      uint32_t b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = __builtin_bit_cast(uint32_t, y[4 * h + i] + 12583040.f);
      w = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
    } else {
      w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], w, true);
    }
    out[h] = w;
  }
  return out;
}

// ---- where things are -------------------------------------------------------------------------------

__device__ __forceinline__ int clamp_page(const int page, const int n_pages) { return min(max(page, 0), n_pages - 1); }

// Byte of the codes where the K rows of (page, tile in page, head) begin; V's are v_step bytes further
template <int D>
__device__ __forceinline__ int64_t tile_at(const Shape8 &s, int page, int tile, int g) {
  const int group = g / s.gg;
  return ((((int64_t)page << (s.log2_T - 5)) + tile) * s.G * 2 + group * 2 * s.gg + (g - group * s.gg)) * (kTile * D);
}
__device__ __forceinline__ int64_t scale_at(const Shape8 &s, int page, int tile, int g) {
  return ((((int64_t)page << (s.log2_T - 5)) + tile) * s.G + g) * 2;
}
template <int D>
__device__ __forceinline__ int64_t tail_at(const Shape8 &s, int row, int kv, int g) {
  return (((int64_t)row * 2 + kv) * s.G + g) * (kTile * D);
}

// Stores of one lane become loads of another of the same wavefront
__device__ __forceinline__ void lanes_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int lds_row(int D) { return D + 8; }      // fp16 numbers from a staged row to the next

// The two operands of 32 fp16 rows: k as K codes are ordered, v as V codes are (through `lds`, 32 * lds_row(D) numbers of the wavefront's own).
// row(kv, key): the row, or NULL for a row of zeros
template <int D>
struct Rows32 {
  half8 k[2][D / 32], v[D / 16];

  template <class Row>
  __device__ __forceinline__ void load(const Row &row, _Float16 *lds, const int lane) {
    const half8 zero = {};
#pragma unroll
    for (int p = 0; p < D / 16; ++p) {
      const int at = p * 64 + lane, key = at / (D / 8), col = at % (D / 8) * 8;
      const _Float16 *from = row(1, key);
      *reinterpret_cast<half8 *>(lds + key * lds_row(D) + col) = from ? *reinterpret_cast<const half8 *>(from + col) : zero;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const _Float16 *from = row(0, 16 * h + lane % 16);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) k[h][c] = from ? *reinterpret_cast<const half8 *>(from + 32 * c + 8 * (lane / 16)) : zero;
    }
    lanes_meet();
#pragma unroll
    for (int e = 0; e < D / 16; ++e)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[e][i] = lds[(4 * (lane / 16) + i + (i < 4 ? 0 : 12)) * lds_row(D) + 16 * e + lane % 16];
    lanes_meet();
  }

  template <int FMT>
  __device__ __forceinline__ void quantise_to(const Cache8 &c, int page, int tile, int g, const int lane) const {
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) mk = fmaxf(mk, largest_of(k[h][i]));
#pragma unroll
    for (int e = 0; e < D / 16; ++e) mv = fmaxf(mv, largest_of(v[e]));
    const float sk = scale_of<FMT>(wave_max(mk)), sv = scale_of<FMT>(wave_max(mv));
    u32x4 *to = reinterpret_cast<u32x4 *>(c.codes + tile_at<D>(c.s, page, tile, g)) + lane;
    u32x4 *to_v = reinterpret_cast<u32x4 *>(reinterpret_cast<uint8_t *>(to) + (int64_t)c.s.gg * kTile * D);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const int h = j / (D / 64), pair = j % (D / 64);
      const u32x2 a = quantise8<FMT>(k[h][2 * pair], sk), b = quantise8<FMT>(k[h][2 * pair + 1], sk);
      to[64 * j] = u32x4{a[0], a[1], b[0], b[1]};
    }
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const u32x2 a = quantise8<FMT>(v[2 * j], sv), b = quantise8<FMT>(v[2 * j + 1], sv);
      to_v[64 * j] = u32x4{a[0], a[1], b[0], b[1]};
    }
    if (lane == 0) *reinterpret_cast<float2 *>(c.scales + scale_at(c.s, page, tile, g)) = make_float2(sk, sv);
  }
};

// ---- storing and reading back -----------------------------------------------------------------------

struct RowsArgs {
  Cache8 c;
  const int32_t *seqs, *starts, *lens;
  _Float16 *k, *v;
  int64_t n_rows, row_stride, layer_stride, codes_layer, scales_layer, tails_layer;
  int32_t batch;
};

// Sequence and tile of work item `item`.  Sequence b's items begin at starts[b] / 32 + 2 b: n rows lie in at most n / 32 + 2 tiles, so
// the items of sequences do not overlap, and no list has to be made.  Two look-ups by all lanes find the sequence among 4096.
__device__ __forceinline__ int sequence_of(const int32_t *starts, const int batch, const int item, const int lane) {
  int first = 0;
  if (batch > 64) {
    const int b = lane * 64;
    first = 64 * max(__popcll(__ballot(b < batch && starts[min(b, batch - 1)] / kTile + 2 * b <= item)) - 1, 0);
  }
  const int b = first + lane;
  return first + max(__popcll(__ballot(b < batch && starts[min(b, batch - 1)] / kTile + 2 * b <= item)) - 1, 0);
}

struct RowsOf {          // the rows of a call that belong to one sequence
  int row, first, n, after, before;      // row of the page table; first row of k / v; rows; tokens after and before
};
__device__ __forceinline__ RowsOf rows_of(const RowsArgs &a, const int b) {
  RowsOf r;
  r.row = min(max(a.seqs ? a.seqs[b] : b, 0), a.c.s.max_seqs - 1);
  r.after = min(max(a.lens[r.row], 0), a.c.s.max_pages << a.c.s.log2_T);
  r.first = min(max(a.starts[b], 0), (int)a.n_rows);
  r.n = min(min(max(a.starts[b + 1], r.first), (int)a.n_rows) - r.first, r.after);
  r.before = r.after - r.n;
  return r;
}

template <int D, int FMT>
__global__ void __launch_bounds__(256) store8_kernel(RowsArgs a) {
  __shared__ _Float16 lds_all[4][kTile * lds_row(D)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (a.c.s.G + 3) >> 2;
  const int item = blockIdx.x / groups, g = (blockIdx.x - item * groups) * 4 + wave;
  if (g >= a.c.s.G || refused(a.c)) return;
  const int b = sequence_of(a.starts, a.batch, item, lane);
  const RowsOf r = rows_of(a, b);
  const int u = item - (a.starts[b] / kTile + 2 * b), t = r.before / kTile + u;
  if (r.n == 0 || u < 0 || t > (r.after - 1) / kTile) return;
  const int64_t layer = blockIdx.y;
  Cache8 c = a.c;
  c.codes += layer * a.codes_layer;
  c.scales += layer * a.scales_layer;
  c.tails += layer * a.tails_layer;
  const _Float16 *const from[2] = {a.k + layer * a.layer_stride + g * D, a.v + layer * a.layer_stride + g * D};
  _Float16 *const tail[2] = {c.tails + tail_at<D>(c.s, r.row, 0, g), c.tails + tail_at<D>(c.s, r.row, 1, g)};
  const auto new_row = [&](int kv, int token) { return from[kv] + (int64_t)(r.first + token - r.before) * a.row_stride; };
  // rows of tile `t` that stay in the tail
  const auto keep = [&](int t) {
    const int lo = max(r.before, t * kTile), n = r.after - lo;
    for (int i = lane; i < 2 * n * (D / 8); i += 64) {
      const int kv = i >= n * (D / 8), at = i - kv * n * (D / 8), token = lo + at / (D / 8), col = at % (D / 8) * 8;
      *reinterpret_cast<half8 *>(tail[kv] + token % kTile * D + col) = *reinterpret_cast<const half8 *>(new_row(kv, token) + col);
    }
  };
  if ((t + 1) * kTile <= r.after) {
    Rows32<D> rows;
    rows.load([&](int kv, int key) -> const _Float16 * {
      const int token = t * kTile + key;
      return token < r.before ? tail[kv] + key * D : new_row(kv, token);
    }, lds_all[wave], lane);
    const int page = clamp_page(c.table[(int64_t)r.row * c.s.max_pages + (t * kTile >> c.s.log2_T)], c.s.n_pages);
    rows.template quantise_to<FMT>(c, page, t & ((1 << (c.s.log2_T - 5)) - 1), g, lane);
    // This tile took rows from the tail: the ones that go there now are stored by the same wavefront, after it has read them
    if (u == 0 && r.before % kTile && r.after % kTile) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      keep(r.after / kTile);
    }
  } else if (u == 0 || r.before % kTile == 0) {
    keep(t);
  }
}

template <int D, int FMT>
__global__ void __launch_bounds__(256) load8_kernel(RowsArgs a) {
  __shared__ _Float16 lds_all[4][kTile * lds_row(D)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (a.c.s.G + 3) >> 2;
  const int item = blockIdx.x / groups, g = (blockIdx.x - item * groups) * 4 + wave;
  if (g >= a.c.s.G) return;
  const int b = sequence_of(a.starts, a.batch, item, lane);
  const RowsOf r = rows_of(a, b);
  const int u = item - (a.starts[b] / kTile + 2 * b), t = r.before / kTile + u;
  if (r.n == 0 || u < 0 || t > (r.after - 1) / kTile) return;
  const int64_t layer = blockIdx.y;
  Cache8 c = a.c;
  c.codes += layer * a.codes_layer;
  c.scales += layer * a.scales_layer;
  c.tails += layer * a.tails_layer;
  _Float16 *const to[2] = {a.k + layer * a.layer_stride + g * D, a.v + layer * a.layer_stride + g * D};
  const auto new_row = [&](int kv, int token) { return to[kv] + (int64_t)(r.first + token - r.before) * a.row_stride; };
  if ((t + 1) * kTile > r.after) {
    const _Float16 *const tail[2] = {c.tails + tail_at<D>(c.s, r.row, 0, g), c.tails + tail_at<D>(c.s, r.row, 1, g)};
    const int lo = max(r.before, t * kTile), n = r.after - lo;
    for (int i = lane; i < 2 * n * (D / 8); i += 64) {
      const int kv = i >= n * (D / 8), at = i - kv * n * (D / 8), token = lo + at / (D / 8), col = at % (D / 8) * 8;
      *reinterpret_cast<half8 *>(new_row(kv, token) + col) = *reinterpret_cast<const half8 *>(tail[kv] + token % kTile * D + col);
    }
    return;
  }
  const int page = clamp_page(c.table[(int64_t)r.row * c.s.max_pages + (t * kTile >> c.s.log2_T)], c.s.n_pages);
  const int tile = t & ((1 << (c.s.log2_T - 5)) - 1);
  const u32x4 *codes = reinterpret_cast<const u32x4 *>(c.codes + tile_at<D>(c.s, page, tile, g)) + lane;
  const u32x4 *codes_v = reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint8_t *>(codes) + (int64_t)c.s.gg * kTile * D);
  const float2 scale = *reinterpret_cast<const float2 *>(c.scales + scale_at(c.s, page, tile, g));
  u32x4 wk[D / 32], wv[D / 32];
#pragma unroll
  for (int j = 0; j < D / 32; ++j) wk[j] = codes[64 * j], wv[j] = codes_v[64 * j];
  const auto value = [](const half8 x, const float s) {
    half8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (_Float16)((float)x[i] * s);
    return y;
  };
  _Float16 *lds = lds_all[wave];
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const half8 y = value(unpack8<FMT>(wv[j][2 * p], wv[j][2 * p + 1]), scale.y);
#pragma unroll
      for (int i = 0; i < 8; ++i) lds[(4 * (lane / 16) + i + (i < 4 ? 0 : 12)) * lds_row(D) + 16 * (2 * j + p) + lane % 16] = y[i];
    }
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const int h = j / (D / 64), token = t * kTile + 16 * h + lane % 16;
    if (token < r.before) continue;
#pragma unroll
    for (int p = 0; p < 2; ++p)
      *reinterpret_cast<half8 *>(new_row(0, token) + 32 * (2 * (j % (D / 64)) + p) + 8 * (lane / 16)) = value(unpack8<FMT>(wk[j][2 * p], wk[j][2 * p + 1]), scale.x);
  }
  lanes_meet();
#pragma unroll
  for (int p = 0; p < D / 16; ++p) {
    const int at = p * 64 + lane, key = at / (D / 8), col = at % (D / 8) * 8, token = t * kTile + key;
    if (token >= r.before) *reinterpret_cast<half8 *>(new_row(1, token) + col) = *reinterpret_cast<const half8 *>(lds + key * lds_row(D) + col);
  }
}

// ---- a step's plan ----------------------------------------------------------------------------------

// What okv8_step_begin leaves in the workspace: the tiles before every sequence, and for every stretch where it begins.
struct Plan8 {
  int32_t *head;           // tiles in all, tiles of a stretch, stretches in use
  int32_t *prefix;         // [batch + 1] whole tiles that are read from codes, before sequence b
  int4 *stretch;           // (sequence, its prefix, the next one's, its row of the page table)
};

constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads) plan8_kernel(const int32_t *seqs, const int32_t *lens, int batch, int appends, Shape8 s,
                                                             int max_stretches, Plan8 plan) {
  __shared__ int prefix[OKV8_MAX_BATCH + 1], sums[kPlanThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  constexpr int kEach = OKV8_MAX_BATCH / kPlanThreads;
  const int each = (batch + kPlanThreads - 1) / kPlanThreads;
  int mine[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = t * each + i;
    int n = 0;
    if (i < each && b < batch) {
      const int row = min(max(seqs ? seqs[b] : b, 0), s.max_seqs - 1);
      n = max(min(lens[row], s.max_pages << s.log2_T) - appends, 0) / kTile;
    }
    mine[i] = n;
    sum += n;
  }
  int upto = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int other = __shfl_up(upto, o);
    if (lane >= o) upto += other;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = upto - sum, total = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = t * each + i;
    if (i >= each || b >= batch) continue;
    prefix[b] = before;
    plan.prefix[b] = before;
    before += mine[i];
  }
  if (t == 0) prefix[batch] = plan.prefix[batch] = total;
  __syncthreads();
  const int span = max((total + max_stretches - 1) / max_stretches, kMinSpan), n = (total + span - 1) / span;
  if (t == 0) plan.head[0] = total, plan.head[1] = span, plan.head[2] = n;
  for (int i = t; i < n; i += kPlanThreads) {
    int lo = 0, hi = batch;              // prefix[lo] <= first tile < prefix[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      (prefix[mid] <= i * span ? lo : hi) = mid;
    }
    plan.stretch[i] = make_int4(lo, prefix[lo], prefix[lo + 1], min(max(seqs ? seqs[lo] : lo, 0), s.max_seqs - 1));
  }
}

// ---- attention --------------------------------------------------------------------------------------

struct Attn8 {
  Cache8 c;
  Plan8 plan;
  const int32_t *seqs, *lens;
  const _Float16 *q, *k_new, *v_new;
  float *part_o, *part_ml;         // partial results by [slot][G][R]; sequence b's tail in slot main_slots + b
  int64_t q_stride, kv_stride;
  int64_t q_layer, kv_layer, codes_layer, scales_layer, tails_layer;      // from a layer's to the next one's
  float scale_log2e;               // log2(e) / sqrt(d)
  int32_t batch, main_slots, main_blocks, layers, appends;      // main_blocks: of a layer
  int32_t slot0;                   // of the layer's partial results
  int32_t max_stretches;           // > 0: no plan was made; up to 64 sequences, whose lengths the wavefronts share out themselves
  void *out;                       // attn8_whole_kernel: [layers][batch][H][d]
  int32_t out_fp32;
};

// The launch covers `layers` layers; a wavefront works for one of them.
__device__ __forceinline__ void of_layer(Attn8 &a, const int layer) {
  a.c.codes += layer * a.codes_layer;
  a.c.scales += layer * a.scales_layer;
  a.c.tails += layer * a.tails_layer;
  a.q += layer * a.q_layer;
  a.k_new += layer * a.kv_layer;
  a.v_new += layer * a.kv_layer;
  a.slot0 = layer * (a.main_slots + a.batch);
}

// The weights that count may be far below the largest: a key that takes most of the softmax and has small values leaves the result to all the others.
// So weights use fp16's whole range (up to 2^15, and at least 2^7 for the largest score when m is raised), and lo, what hi leaves of one, is 2^10
// times larger than it and rounded to nearest: a weight is off by 2^-22 of itself or by 2^-35, whichever is more, and 2^-35 is at most 2^-42 of
// the largest.  (With lo in hi's sums its grid is fp16's, 2^-24, and cutting off there, one way, took 7e-3 off the result of 16384 keys
// whose scores are 12 below one key's of small values; now 1.1e-6.)
template <int D>
struct Softmax8 {
  static constexpr float kTop = 15.f, kRaised = 7.f, kLo = 1024.f;
  floatx4 o[D / 16], o_lo[D / 16];         // of hi; of lo, kLo times too large
  float m, l;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < D / 16; ++e) o[e] = o_lo[e] = floatx4{0.f, 0.f, 0.f, 0.f};
    m = -__builtin_inff(), l = 0.f;
  }

  // The lane's 8 scores of 32 keys, in log2 units and with log2 of the tile's V scale added -> weights w = 2^(s - m) as two fp16 numbers each.
  // The scale is in the weights, so that the products add up in the accumulators of the matrix cores;
  // l counts the weights without it.  m is raised, and what is there multiplied down, only when a weight would pass 2^15, 8 above
  // the largest score that m was raised for: hardly ever after a piece's first tile.
  // FIRST: nothing is there yet.  Then m tells even from scores that are all -infinity that there were keys (their weights are 0 and not NaN: other
  // pieces of the sequence may have more).
  template <bool FIRST = false>
  __device__ __forceinline__ void weigh(const float (&s)[8], half8 &hi, half8 &lo, const float scale) {
    const float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    if constexpr (FIRST) {
      m = fmaxf(max_with_lane_xor<16>(max_with_lane_xor<32>(top)) - kRaised, -__FLT_MAX__);
    } else if (__any(top > m + kTop)) {
      const float now = fmaxf(m, max_with_lane_xor<16>(max_with_lane_xor<32>(top)) - kRaised);
      const float alpha = m == now ? 1.f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= alpha;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) o[e] *= alpha, o_lo[e] *= alpha;
    }
    float w[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = __builtin_amdgcn_exp2f(s[i] - m);
      sum += w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const half2v h = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[i], w[i + 1]));
      hi[i] = h[0], hi[i + 1] = h[1];
      lo[i] = (_Float16)((w[i] - (float)h[0]) * kLo), lo[i + 1] = (_Float16)((w[i + 1] - (float)h[1]) * kLo);
    }
    l = fmaf(sum, scale, l);
  }
  __device__ __forceinline__ floatx4 sum_of(const int e) const { return o[e] + o_lo[e] * (1.f / kLo); }
  __device__ __forceinline__ void add(const int e, const half8 v, const half8 hi, const half8 lo) {
    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, hi, o[e], 0, 0, 0);
    o_lo[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, lo, o_lo[e], 0, 0, 0);
  }
  // The same of the first keys, whose values may be infinite: a weight that hi has whole leaves lo 0, whose product with an infinity would be NaN.  (Infinities and NaN
  // reach the sums by hi, and are the largest finite number in lo's.)
  __device__ __forceinline__ void first(const int e, const half8 v, const half8 hi, const half8 lo) {
    const half8 most = (half8)(_Float16)65504.f;
    const floatx4 none = {0.f, 0.f, 0.f, 0.f};
    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, hi, none, 0, 0, 0);
    o_lo[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_elementwise_max(__builtin_elementwise_min(v, most), -most), lo, none, 0, 0, 0);
    // (one sum leaves registers to the tile that is under way beside a tail: at d = 64 four wavefronts a SIMD and not three; at 128 it is slower)
    if constexpr (D == 64) o[e] = sum_of(e), o_lo[e] = none;
  }
  __device__ __forceinline__ void write(const Attn8 &a, const int64_t slot, const int g, const int lane) const {
    const float sum = sum_with_lane_xor<16>(sum_with_lane_xor<32>(l));
    const int R = a.c.s.R, r = lane % 16;
    if (r >= R) return;
    const int64_t at = ((a.slot0 + slot) * a.c.s.G + g) * R + r;
    if (lane < 16) *reinterpret_cast<float2 *>(a.part_ml + 2 * at) = make_float2(m, sum);
#pragma unroll
    for (int e = 0; e < D / 16; ++e) *reinterpret_cast<floatx4 *>(a.part_o + at * D + 16 * e + 4 * (lane / 16)) = sum_of(e);
  }
};

template <int D>
__device__ __forceinline__ void load_q(half8 (&q)[D / 32], const Attn8 &a, const int b, const int g, const int lane) {
  const int r = lane % 16;
  const half8 zero = {};
  const _Float16 *from = a.q + b * a.q_stride + (int64_t)(g * a.c.s.R + r) * D + 8 * (lane / 16);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) q[c] = r < a.c.s.R ? *reinterpret_cast<const half8 *>(from + 32 * c) : zero;
}

// What a step reads of a sequence: `held` keys in codes, `rows` in the tail
struct Keys8 {
  int row, held, rows;
};
__device__ __forceinline__ Keys8 keys_of(const Attn8 &a, const int b) {
  const Shape8 &s = a.c.s;
  Keys8 k;
  k.row = min(max(a.seqs ? a.seqs[b] : b, 0), s.max_seqs - 1);
  const int n = min(max(a.lens[k.row], 0), s.max_pages << s.log2_T);
  k.held = max(n - a.appends, 0) / kTile * kTile;
  k.rows = n - k.held;
  return k;
}

// A sequence's fp16 tail: the appended row goes there, its keys are attended (the first ones of `acc`), and it is quantised when it is full.
template <int D, int FMT>
__device__ __forceinline__ void attend_tail(Softmax8<D> &acc, const half8 (&q)[D / 32], const Attn8 &a, const Keys8 &keys, const int b, const int g,
                                            _Float16 *lds, const int lane) {
  const Shape8 &s = a.c.s;
  const int row = keys.row, held = keys.held, rows = keys.rows;
  if (rows > 0) {
    // (where a full tail goes: asked for before the rows, so that it is there when they are attended)
    const bool full = a.appends && rows == kTile, writes = a.appends && !refused(a.c);
    const int to_page = full ? a.c.table[(int64_t)row * s.max_pages + (held >> s.log2_T)] : 0;
    _Float16 *const tail[2] = {a.c.tails + tail_at<D>(s, row, 0, g), a.c.tails + tail_at<D>(s, row, 1, g)};
    const _Float16 *const fresh[2] = {a.k_new + b * a.kv_stride + g * D, a.v_new + b * a.kv_stride + g * D};
    Rows32<D> x;
    x.load([&](int kv, int key) -> const _Float16 * {
      return key >= rows ? nullptr : a.appends && key == rows - 1 ? fresh[kv] : tail[kv] + key * D;
    }, lds, lane);
    if (writes && lane < 2 * (D / 8)) {
      const int kv = lane / (D / 8), col = lane % (D / 8) * 8;
      *reinterpret_cast<half8 *>(tail[kv] + (rows - 1) * D + col) = *reinterpret_cast<const half8 *>(fresh[kv] + col);
    }
    float score[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      floatx4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < D / 32; ++c) t = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.k[h][c], q[c], t, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) score[4 * h + i] = 16 * h + 4 * (lane / 16) + i < rows ? t[i] * a.scale_log2e : -__builtin_inff();
    }
    half8 hi, lo;
    acc.template weigh<true>(score, hi, lo, 1.f);
#pragma unroll
    for (int e = 0; e < D / 16; ++e) acc.first(e, x.v[e], hi, lo);
    if (full && writes) x.template quantise_to<FMT>(a.c, clamp_page(to_page, s.n_pages), (held / kTile) & ((1 << (s.log2_T - 5)) - 1), g, lane);
  }
}

template <int D, bool NT>
__device__ __forceinline__ void load_codes(u32x4 (&w)[D / 32], const uint8_t *from) {
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const u32x4 *p = reinterpret_cast<const u32x4 *>(from) + 64 * j;
    w[j] = NT ? __builtin_nontemporal_load(p) : *p;
  }
}

// A tile's codes and scales
template <int D>
struct Tile8 {
  u32x4 k[D / 32], v[D / 32];
  float2 scale;
};
template <int D, int FMT>
__device__ __forceinline__ void reduce_tile(Softmax8<D> &acc, const half8 (&q)[D / 32], const Tile8<D> &tile, const float scale_log2e) {
  float score[8];
  // A tile of zeros (scale 0, codes 0) has any scale, and takes one far below all others (at least 2^-33): m, which its scores may raise, would
  // otherwise leave the other tiles' weights too few bits.  What it adds to l is at most 2^48 2^15 a key.
  const float scale_v = tile.scale.y == 0.f ? 0x1p-48f : tile.scale.y, by = tile.scale.x * scale_log2e, log2_v = __builtin_amdgcn_logf(scale_v);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const u32x4 w = tile.k[h * (D / 64) + c / 2];
      x = __builtin_amdgcn_mfma_f32_16x16x32_f16(unpack8<FMT>(w[2 * (c % 2)], w[2 * (c % 2) + 1]), q[c], x, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) score[4 * h + j] = fmaf(x[j], by, log2_v);
  }
  half8 hi, lo;
  acc.weigh(score, hi, lo, __builtin_amdgcn_rcpf(scale_v));
#pragma unroll
  for (int e = 0; e < D / 16; ++e) acc.add(e, unpack8<FMT>(tile.v[e / 2][2 * (e % 2)], tile.v[e / 2][2 * (e % 2) + 1]), hi, lo);
}

template <int D, int FMT, bool NT>
__global__ void __launch_bounds__(256) attn8_kernel(const Attn8 launch) {
  __shared__ _Float16 lds_all[4][kTile * lds_row(D)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Attn8 a = launch;
  // the layers' code readers first, then their tails, which take the places beside them
  int block = blockIdx.x;
  if (block >= a.main_blocks * a.layers) {
    block -= a.main_blocks * a.layers;
    const int per_layer = (a.batch * a.c.s.G + 3) >> 2, layer = block / per_layer;
    of_layer(a, layer);
    const int unit = (block - layer * per_layer) * 4 + wave, b = unit / a.c.s.G, g = unit - b * a.c.s.G;
    if (b >= a.batch) return;
    half8 q[D / 32];
    Softmax8<D> acc;
    load_q<D>(q, a, b, g, lane);
    acc.clear();
    attend_tail<D, FMT>(acc, q, a, keys_of(a, b), b, g, lds_all[wave], lane);
    acc.write(a, a.main_slots + b, g, lane);
    return;
  }
  const Shape8 s = a.c.s;
  const int layer = block / a.main_blocks, unit = (block - layer * a.main_blocks) * 4 + wave, str = unit / s.G, g = unit - str * s.G;
  of_layer(a, layer);
  // The plan, or, for a step of up to 64 sequences, what plan8_kernel does with a lane per sequence: `upto` tiles with that of the lane, `row_of` its
  // row of the table, `there` the sequences that have tiles.  It costs a launch 1 us and saves one of 2.6 to 4.7; the launch that
  // joins the results finds the plan where plan8_kernel leaves it.
  const bool own_plan = a.max_stretches > 0;
  int upto = 0, row_of = 0, total, span;
  uint64_t there = 0;
  int4 begin;
  if (own_plan) {
    row_of = min(max(a.seqs && lane < a.batch ? a.seqs[lane] : lane, 0), s.max_seqs - 1);
    const int tiles = lane < a.batch ? max(min(a.lens[row_of], s.max_pages << s.log2_T) - a.appends, 0) / kTile : 0;
    there = __ballot(tiles > 0);
    upto = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int other = __shfl_up(upto, o);
      if (lane >= o) upto += other;
    }
    total = __builtin_amdgcn_readlane(upto, 63);
    span = max((total + a.max_stretches - 1) / a.max_stretches, kMinSpan);
    if (blockIdx.x == 0 && wave == 0) {
      if (lane < a.batch) a.plan.prefix[lane + 1] = upto;
      if (lane == 0) a.plan.prefix[0] = 0, a.plan.head[1] = span;
    }
    if (str * span >= total) return;
    const int first = __popcll(__ballot(upto <= str * span));
    begin = make_int4(first, first ? __builtin_amdgcn_readlane(upto, first - 1) : 0, __builtin_amdgcn_readlane(upto, first),
                      __builtin_amdgcn_readlane(row_of, first));
  } else {
    total = a.plan.head[0], span = a.plan.head[1];
    if (str * span >= total) return;
    begin = a.plan.stretch[str];
  }
  const int log2_tpp = s.log2_T - 5;
  const int64_t head_at = tile_at<D>(s, 0, 0, g) + 16 * lane;
  const int64_t tile_bytes = (int64_t)s.G * 2 * kTile * D;
  const int v_step = s.gg * kTile * D;

  // where the loads are: tile `next` of sequence fb (row frow of the table), `f_left` more of it in this stretch, `ahead` of all
  const int t0 = str * span;
  int left = min(span, total - t0), ahead = left;
  int fb = begin.x, frow = begin.w, next = t0 - begin.y, in_seq = min(begin.z - t0, left), f_left = in_seq, pages, page0;
  const auto look_up = [&]() {
    page0 = next >> log2_tpp;
    pages = clamp_page(a.c.table[(int64_t)frow * s.max_pages + min(page0 + lane, s.max_pages - 1)], s.n_pages);
  };
  look_up();
  // the sequence after it: where it is takes three dependent loads, which are under way while this one's tiles are
  int then_b = 0, then_row = 0, then_tiles = 0, then_pages = 0;
  const auto look_ahead = [&](const int more) {      // `more` tiles of the stretch behind fb's
    if (more <= 0) return;
    int lo, hi;
    if (own_plan) {
      then_b = __builtin_ctzll(there & (~0ull << fb << 1));
      lo = __builtin_amdgcn_readlane(upto, then_b - 1), hi = __builtin_amdgcn_readlane(upto, then_b);
      then_row = __builtin_amdgcn_readlane(row_of, then_b);
    } else {
      then_b = fb;
      do {
        ++then_b;
        lo = a.plan.prefix[then_b], hi = a.plan.prefix[then_b + 1];
      } while (lo == hi);
      then_row = min(max(a.seqs ? a.seqs[then_b] : then_b, 0), s.max_seqs - 1);
    }
    then_tiles = min(hi - lo, more);
    then_pages = clamp_page(a.c.table[(int64_t)then_row * s.max_pages + min(lane, s.max_pages - 1)], s.n_pages);
  };
  const uint8_t *at;
  const float *scale_from;
  const auto place = [&]() {
    const int p = next >> log2_tpp;
    if (p - page0 >= 64) look_up();
    const int64_t tile = ((int64_t)__builtin_amdgcn_readlane(pages, p - page0) << log2_tpp) + (next & ((1 << log2_tpp) - 1));
    at = a.c.codes + tile * tile_bytes + head_at;
    scale_from = a.c.scales + (tile * s.G + g) * 2;
  };

  struct Buffer : Tile8<D> {
    int b, tiles;                                // its sequence, and that one's tiles in this stretch
  };
  // A tile's K and V are asked for together, when the one before has been reduced: K as soon as its registers are free and V later is 9 % slower
  // (ragged grouped heads 437 us a case against 397), a second tile in flight no faster (401).
  const auto fetch = [&](Buffer &t) {
    if (ahead == 0) return;
    place();
    load_codes<D, NT>(t.k, at);
    load_codes<D, NT>(t.v, at + v_step);
    t.scale = *reinterpret_cast<const float2 *>(scale_from);
    t.b = fb, t.tiles = in_seq;
    --ahead;
    ++next;
    if (--f_left == 0 && ahead > 0) {            // the next tile is another sequence's
      fb = then_b, frow = then_row, pages = then_pages;
      next = page0 = 0;
      f_left = in_seq = then_tiles;
      look_ahead(ahead - in_seq);
    }
  };
  Buffer tile;
  look_ahead(ahead - in_seq);
  fetch(tile);
  int b = tile.b, piece = tile.tiles;            // sequence at hand, tiles of it to go
  half8 q[D / 32];
  Softmax8<D> acc;
  load_q<D>(q, a, b, g, lane);
  acc.clear();
  for (;;) {
    reduce_tile<D, FMT>(acc, q, tile, a.scale_log2e);
    fetch(tile);
    if (--piece == 0) {
      acc.write(a, str + b, g, lane);
      if (left > 1) {
        b = tile.b, piece = tile.tiles;
        load_q<D>(q, a, b, g, lane);
        acc.clear();
      }
    }
    if (--left == 0) break;
  }
}

// A launch over sequences that are short, without a second one that joins: a workgroup has a whole (layer, sequence, KV head), its wavefronts take the
// tiles in turn, the one with the fewest also the tail, and join through LDS.  Bound by its chain of dependent loads (length and table, codes, LDS).
// When: see whole_waves().
template <int D, int FMT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) attn8_whole_kernel(const Attn8 launch) {
  __shared__ floatx4 o_all[WAVES][D / 16][64];
  __shared__ float ml_all[WAVES][2][16];
  __shared__ _Float16 lds[kTile * lds_row(D)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Attn8 a = launch;
  const Shape8 s = a.c.s;
  const int item = blockIdx.x / s.G, g = blockIdx.x - item * s.G, layer = item / a.batch, b = item - layer * a.batch;
  of_layer(a, layer);
  const Keys8 keys = keys_of(a, b);
  const int tiles = keys.held / kTile, log2_tpp = s.log2_T - 5;
  const int pages = clamp_page(a.c.table[(int64_t)keys.row * s.max_pages + min(lane, s.max_pages - 1)], s.n_pages);      // (at most 64 of them)
  Tile8<D> tile;
  const auto fetch = [&](const int t) {
    const int64_t at = ((int64_t)__builtin_amdgcn_readlane(pages, t >> log2_tpp) << log2_tpp) + (t & ((1 << log2_tpp) - 1));
    const uint8_t *from = a.c.codes + at * s.G * 2 * kTile * D + tile_at<D>(s, 0, 0, g) + 16 * lane;
    load_codes<D, false>(tile.k, from);
    load_codes<D, false>(tile.v, from + s.gg * kTile * D);
    tile.scale = *reinterpret_cast<const float2 *>(a.c.scales + (at * s.G + g) * 2);
  };
  half8 q[D / 32];
  Softmax8<D> acc;
  acc.clear();
  load_q<D>(q, a, b, g, lane);
  if (wave < tiles) fetch(wave);
  if (wave == tiles % WAVES) attend_tail<D, FMT>(acc, q, a, keys, b, g, lds, lane);
  for (int t = wave; t < tiles; t += WAVES) {
    reduce_tile<D, FMT>(acc, q, tile, a.scale_log2e);
    if (t + WAVES < tiles) fetch(t + WAVES);
  }
  const float sum = sum_with_lane_xor<16>(sum_with_lane_xor<32>(acc.l));
  if (lane < 16) ml_all[wave][0][lane] = acc.m, ml_all[wave][1][lane] = sum;
#pragma unroll
  for (int e = 0; e < D / 16; ++e) o_all[wave][e][lane] = acc.sum_of(e);
  __syncthreads();
  // 4 consecutive elements of a query head per thread
  for (int i = threadIdx.x; i < D / 16 * 64; i += 64 * WAVES) {
    const int e = i >> 6, l = i & 63, r = l % 16;
    if (r >= s.R) continue;
    float top = ml_all[0][0][r], all = 0.f;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, ml_all[w][0][r]);
    const float base = top == -__builtin_inff() ? 0.f : top;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float by = __builtin_amdgcn_exp2f(ml_all[w][0][r] - base);
      all = fmaf(by, ml_all[w][1][r], all);
      o += by * o_all[w][e][l];
    }
    o *= all == 0.f && top == -__builtin_inff() ? 0.f : 1.f / all;      // no key at all: 0
    const int64_t to = ((int64_t)item * s.G * s.R + g * s.R + r) * D + 16 * e + 4 * (l / 16);
    if (a.out_fp32) *reinterpret_cast<floatx4 *>(static_cast<float *>(a.out) + to) = o;
    else *reinterpret_cast<half4 *>(static_cast<_Float16 *>(a.out) + to) = half4{(_Float16)o[0], (_Float16)o[1], (_Float16)o[2], (_Float16)o[3]};
  }
}

struct Merge8 {
  Plan8 plan;
  const float *part_o, *part_ml;
  void *out;                       // [layers][batch][H][d]
  int32_t batch, H, main_slots, layers, out_fp32;
};

// out = sum_p w_p o_p / sum_p w_p l_p with w_p = 2^(m_p - max m) over a row's pieces.  WAVES wavefronts share a row's pieces: 1, four rows to a
// workgroup, where most sequences are cut little; 4 where there are few sequences and therefore many pieces of each.
template <int D, int WAVES>
__global__ void __launch_bounds__(256) merge8_kernel(Merge8 a) {
  constexpr int E = D / 64, kJoin = WAVES == 1 ? 4 : 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x, share = WAVES == 1 ? 0 : wave;
  if (row >= a.layers * a.batch * a.H) return;
  const int seq = row / a.H, h = row - seq * a.H, layer = seq / a.batch, b = seq - layer * a.batch;
  const int slot0 = layer * (a.main_slots + a.batch);
  const int span = a.plan.head[1], lo = a.plan.prefix[b], hi = a.plan.prefix[b + 1];
  const int first = lo / span, pieces = (hi > lo ? (hi - 1) / span - first + 1 : 0) + 1;      // the last one is the tail's
  const auto at = [&](int p) { return (int64_t)(slot0 + (p == pieces - 1 ? a.main_slots + b : first + p + b)) * a.H + h; };
  float top = -__builtin_inff(), sum = 0.f, o[E] = {};
  for (int p0 = share * 64; p0 < pieces; p0 += 64 * WAVES) {
    const int n = min(64, pieces - p0);
    float x[kJoin][E];                                     // kJoin pieces at a time are in flight, the first with the maxima and sums of all
    const auto ask = [&](const int i) {
#pragma unroll
      for (int j = 0; j < kJoin; ++j) {
        // (beyond the last piece the first one: if that is no tail, it is finite, or NaN as the result will be, and its weight here, 0, adds nothing)
        const float *from = a.part_o + at(p0 + (i + j < n ? i + j : 0)) * D + E * lane;
#pragma unroll
        for (int e = 0; e < E; ++e) x[j][e] = from[e];
      }
    };
    const float2 ml = lane < n ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * at(p0 + lane)) : make_float2(-__builtin_inff(), 0.f);
    ask(0);
    const float now = fmaxf(top, wave_max(ml.x)), base = now == -__builtin_inff() ? 0.f : now;
    const float w = __builtin_amdgcn_exp2f(ml.x - base), old = __builtin_amdgcn_exp2f(top - base);
    top = now;
    sum = sum * old + wave_sum(w * ml.y);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= old;
    if (n == 1) {                                          // a tail, which may be infinite
      const float w0 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), 0));
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(w0, x[0][e], o[e]);
      continue;
    }
    for (int i = 0; i < n; i += kJoin) {
      if (i) ask(i);
#pragma unroll
      for (int j = 0; j < kJoin; ++j) {
        const float wi = i + j < n ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), min(i + j, n - 1))) : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(wi, x[j][e], o[e]);
      }
    }
  }
  if constexpr (WAVES > 1) {
    __shared__ float all[WAVES][2 + D];
    if (lane == 0) all[wave][0] = top, all[wave][1] = sum;
#pragma unroll
    for (int e = 0; e < E; ++e) all[wave][2 + E * lane + e] = o[e];
    __syncthreads();
    if (wave) return;
    const float own = top;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = fmaxf(top, all[i][0]);
    const float base = top == -__builtin_inff() ? 0.f : top;
    const float w0 = __builtin_amdgcn_exp2f(own - base);
    sum *= w0;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= w0;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) {
      const float w = __builtin_amdgcn_exp2f(all[i][0] - base);
      sum = fmaf(w, all[i][1], sum);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(w, all[i][2 + E * lane + e], o[e]);
    }
  }
  const float by = sum == 0.f && top == -__builtin_inff() ? 0.f : 1.f / sum;      // no key at all: 0
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t to = (int64_t)row * D + E * lane + e;
    if (a.out_fp32) static_cast<float *>(a.out)[to] = o[e] * by;
    else static_cast<_Float16 *>(a.out)[to] = (_Float16)(o[e] * by);
  }
}

// ---- host -------------------------------------------------------------------------------------------

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

const char *shape_problem(const okv8_cache *c) {
  if (!c) return "cache is NULL";
  if (c->n_layers < 1) return "n_layers must be at least 1";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "n_kv_heads must be in [1, 1024]";
  if (c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 16) return "n_q_heads must be 1 to 16 times n_kv_heads";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->page_tokens < kTile || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1))) return "page_tokens must be a power of two in [32, 1024]";
  if (c->format != OKV8_INT8 && c->format != OKV8_E4M3) return "format must be OKV8_INT8 or OKV8_E4M3";
  if (c->out_dtype != 0 && c->out_dtype != 1) return "out_dtype must be 0 (fp16) or 1 (fp32)";
  if (c->max_seqs < 1 || c->max_pages_per_seq < 1) return "max_seqs and max_pages_per_seq must be at least 1";
  if ((int64_t)c->max_pages_per_seq * c->page_tokens > 0x7fffffff - 4 * kTile) return "max_pages_per_seq * page_tokens must be below 2^31 - 128";
  if (c->n_pages < 1 || c->n_pages > 0x7fffffff) return "n_pages must be in [1, 2^31 - 1]";
  return nullptr;
}
const char *cache_problem(const okv8_cache *c) {
  if (const char *why = shape_problem(c)) return why;
  if (!c->codes || !c->scales || !c->tails || !c->page_table) return "NULL buffer";
  if (!aligned16(c->codes) || !aligned16(c->scales) || !aligned16(c->tails)) return "buffers must be 16-byte aligned";
  return nullptr;
}

int log2_of(int32_t x) { return 31 - __builtin_clz((unsigned)x); }
int64_t codes_layer_bytes(const okv8_cache *c) { return c->n_pages * c->page_tokens * 2 * c->n_kv_heads * c->head_dim; }
int64_t scales_layer_floats(const okv8_cache *c) { return c->n_pages * (c->page_tokens / kTile) * 2 * c->n_kv_heads; }
int64_t tails_layer_halves(const okv8_cache *c) { return (int64_t)c->max_seqs * 2 * c->n_kv_heads * kTile * c->head_dim; }

Cache8 cache_of(const okv8_cache *c, int32_t layer) {
  Cache8 k;
  k.codes = static_cast<uint8_t *>(c->codes) + layer * codes_layer_bytes(c);
  k.scales = static_cast<float *>(c->scales) + layer * scales_layer_floats(c);
  k.tails = static_cast<_Float16 *>(c->tails) + layer * tails_layer_halves(c);
  k.table = c->page_table, k.refused = c->refused;
  k.s = {c->n_kv_heads, c->n_q_heads / c->n_kv_heads, kv_head_group(c->n_kv_heads, c->head_dim), log2_of(c->page_tokens),
         c->max_seqs, c->max_pages_per_seq, (int32_t)c->n_pages};
  return k;
}

// Stretches of a launch that covers this many layers: a wavefront for each (layer, stretch, KV head)
int max_stretches(const okv8_cache *c, int layers) { return std::max(1, (c->head_dim == 64 ? 2 : 1) * kWaves / (c->n_kv_heads * layers)); }

// The workspace: plan (head, prefix, stretches), then for every layer of a launch the partial results of batch + stretches slots and of batch tails.
struct Workspace8 {
  int64_t prefix, stretch, ml, o, bytes;
  int32_t slots, layers, stretches;
};
Workspace8 workspace_of(const okv8_cache *c, int32_t batch, int32_t layers) {
  const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
  Workspace8 w;
  w.layers = layers;
  w.stretches = max_stretches(c, layers);
  w.slots = batch + w.stretches;
  w.prefix = 256;
  w.stretch = up(w.prefix + 4 * (int64_t)(batch + 1));
  w.ml = up(w.stretch + 16 * (int64_t)w.stretches);
  const int64_t rows = (int64_t)layers * (w.slots + batch) * c->n_q_heads;
  w.o = up(w.ml + 8 * rows);
  w.bytes = up(w.o + 4 * rows * c->head_dim);
  return w;
}

// Layers that okv8_decode_step attends in one launch: all of them, up to 32, where the workspace holds their partial results
constexpr int kLayersAbreast = 32;
Workspace8 workspace_for(const okv8_cache *c, const okv8_step *s) {
  int layers = std::min(c->n_layers, kLayersAbreast);
  while (layers > 1 && workspace_of(c, s->batch, layers).bytes > s->workspace_bytes) --layers;
  return workspace_of(c, s->batch, layers);
}

Plan8 plan_of(const Workspace8 &w, void *base) {
  char *p = static_cast<char *>(base);
  return {reinterpret_cast<int32_t *>(p), reinterpret_cast<int32_t *>(p + w.prefix), reinterpret_cast<int4 *>(p + w.stretch)};
}

int step_problem(const char *who, const okv8_cache *c, const okv8_step *s) {
  if (const char *why = cache_problem(c)) return report(OKV_EINVAL, "%s: %s", who, why);
  if (!s) return report(OKV_EINVAL, "%s: step is NULL", who);
  if (s->batch < 1 || s->batch > OKV8_MAX_BATCH || s->batch > c->max_seqs)
    return report(OKV_EINVAL, "%s: batch must be in [1, min(max_seqs, %d)]", who, OKV8_MAX_BATCH);
  if ((int64_t)s->batch * c->max_pages_per_seq * (c->page_tokens / kTile) > 0x70000000)
    return report(OKV_EINVAL, "%s: batch * max_pages_per_seq * page_tokens is beyond what is counted in 32 bits", who);
  if (s->appends != 0 && s->appends != 1) return report(OKV_EINVAL, "%s: appends must be 0 or 1", who);
  if (!s->lens || !s->workspace) return report(OKV_EINVAL, "%s: NULL pointer", who);
  if (reinterpret_cast<uintptr_t>(s->workspace) & 255) return report(OKV_EINVAL, "%s: the workspace must be 256-byte aligned", who);
  if (s->workspace_bytes < workspace_of(c, s->batch, 1).bytes)
    return report(OKV_ENOSPC, "%s: the workspace has %lld bytes, %lld are needed", who, (long long)s->workspace_bytes, (long long)workspace_of(c, s->batch, 1).bytes);
  return OKV_OK;
}

int hip_result(const char *who, hipError_t e) { return e == hipSuccess ? OKV_OK : report(OKV_EHIP, "%s: %s", who, hipGetErrorString(e)); }

template <template <int, int> class Launch, class... Args>
void by_format(const okv8_cache *c, Args... args) {
  if (c->head_dim == 128) c->format == OKV8_INT8 ? Launch<128, OKV8_INT8>::go(args...) : Launch<128, OKV8_E4M3>::go(args...);
  else c->format == OKV8_INT8 ? Launch<64, OKV8_INT8>::go(args...) : Launch<64, OKV8_E4M3>::go(args...);
}
template <int D, int FMT>
struct StoreLaunch {
  static void go(const RowsArgs &a, dim3 grid, hipStream_t stream) { hipLaunchKernelGGL((store8_kernel<D, FMT>), grid, dim3(256), 0, stream, a); }
};
template <int D, int FMT>
struct LoadLaunch {
  static void go(const RowsArgs &a, dim3 grid, hipStream_t stream) { hipLaunchKernelGGL((load8_kernel<D, FMT>), grid, dim3(256), 0, stream, a); }
};
template <int D, int FMT>
struct AttnLaunch8 {
  static void go(const Attn8 &a, dim3 grid, bool nt, hipStream_t stream) {
    if (nt) hipLaunchKernelGGL((attn8_kernel<D, FMT, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((attn8_kernel<D, FMT, false>), grid, dim3(256), 0, stream, a);
  }
};

template <int D, int FMT>
struct WholeLaunch8 {
  static void go(const Attn8 &a, dim3 grid, int waves, hipStream_t stream) {
    if (waves == 8) hipLaunchKernelGGL((attn8_whole_kernel<D, FMT, 8>), grid, dim3(512), 0, stream, a);
    else hipLaunchKernelGGL((attn8_whole_kernel<D, FMT, 4>), grid, dim3(256), 0, stream, a);
  }
};

int rows_call(const char *who, bool store, const okv8_cache *c, int32_t layer, int32_t n_layers, int32_t batch, const int32_t *seqs,
              const int32_t *starts, const int32_t *lens, int64_t n_rows, const void *k, const void *v, int64_t row_stride,
              int64_t layer_stride, void *stream) {
  if (const char *why = cache_problem(c)) return report(OKV_EINVAL, "%s: %s", who, why);
  if (layer < 0 || n_layers < 1 || n_layers > c->n_layers - layer) return report(OKV_EINVAL, "%s: layers out of range", who);
  if (batch < 1 || batch > OKV8_MAX_BATCH || batch > c->max_seqs) return report(OKV_EINVAL, "%s: batch must be in [1, min(max_seqs, %d)]", who, OKV8_MAX_BATCH);
  if (!starts || !lens) return report(OKV_EINVAL, "%s: NULL pointer", who);
  if (n_rows < 0 || n_rows > 0x7fffffff - 64 * OKV8_MAX_BATCH) return report(OKV_EINVAL, "%s: bad n_rows", who);
  if (n_rows == 0) return OKV_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return report(OKV_EINVAL, "%s: NULL or misaligned pointer", who);
  if (row_stride < (int64_t)c->n_kv_heads * c->head_dim || row_stride % 8 || layer_stride % 8 || (n_layers > 1 && layer_stride < 0))
    return report(OKV_EINVAL, "%s: strides must be multiples of 8, a row's at least n_kv_heads * head_dim", who);
  const int64_t blocks = (n_rows / kTile + 2 * (int64_t)batch) * ((c->n_kv_heads + 3) / 4);
  if (blocks > 0x7fffffff || n_layers > 65535) return report(OKV_EINVAL, "%s: too many rows for one call", who);
  RowsArgs a;
  a.c = cache_of(c, layer);
  a.seqs = seqs, a.starts = starts, a.lens = lens;
  a.k = static_cast<_Float16 *>(const_cast<void *>(k)), a.v = static_cast<_Float16 *>(const_cast<void *>(v));
  a.n_rows = n_rows, a.row_stride = row_stride, a.layer_stride = layer_stride;
  a.codes_layer = codes_layer_bytes(c), a.scales_layer = scales_layer_floats(c), a.tails_layer = tails_layer_halves(c);
  a.batch = batch;
  const dim3 grid((unsigned)blocks, (unsigned)n_layers);
  if (store) by_format<StoreLaunch>(c, a, grid, static_cast<hipStream_t>(stream));
  else by_format<LoadLaunch>(c, a, grid, static_cast<hipStream_t>(stream));
  return hip_result(who, hipGetLastError());
}

// Codes that do not fit the memory-side cache (256 MiB) are read past it, so that they do not push out what is used again.
bool streamed(const okv8_cache *c) { return codes_layer_bytes(c) * c->n_layers > (int64_t)256 << 20; }

// Wavefronts of the workgroups that attend a whole sequence and KV head each, 0: the sequences are cut.  Lengths are on the GPU, so the rule goes by
// what a row of the page table can hold: at most 1024 keys (a lane has a page), so that a long sequence among short ones costs little.
// us a step cut / 4 / 8 wavefronts: 4 x 250..256 keys x 8 KV heads, d = 64, 8.0 / 5.0 / 5.0; 16 x 100..400 x 12, d = 128, 10.0 / 7.2 / 6.7;
// 4 x 1000..1024 x 32, d = 128, 13.3 / 13.4 / 10.9; 100 x 10..200 x 8, d = 64, 11.9 / 6.2 / 8.6; 64 x 400..512 x 8, d = 128, 17.8 / 15.8 /
// 19.1; and where it is not taken: 32 x 700..768 x 32, d = 128, 34.9 / 36.6 / 41.8; 1 x 2000 x 4, d = 64, 8.9 / 11.6 / 9.9.
int whole_waves(const okv8_cache *c, int32_t batch, int32_t layers) {
  const int64_t keys = (int64_t)c->max_pages_per_seq * c->page_tokens, groups = (int64_t)layers * batch * c->n_kv_heads;
  if (keys > 1024) return 0;
  return groups <= 256 ? 8 : groups <= 1024 && groups * keys <= 1 << 19 ? 4 : 0;
}

// w.layers layers from `layer` on, as far as there are
int attend(const char *who, const okv8_cache *c, const okv8_step *s, const Workspace8 &w, bool planned, int32_t layer, int32_t layers, const void *q, int64_t q_stride,
           const void *k_new, const void *v_new, int64_t kv_stride, void *out) {
  char *base = static_cast<char *>(s->workspace);
  const hipStream_t stream = static_cast<hipStream_t>(s->stream);
  Attn8 a;
  a.c = cache_of(c, layer);
  a.plan = plan_of(w, base);
  a.seqs = s->seqs, a.lens = s->lens;
  a.q = static_cast<const _Float16 *>(q), a.k_new = static_cast<const _Float16 *>(k_new), a.v_new = static_cast<const _Float16 *>(v_new);
  a.part_ml = reinterpret_cast<float *>(base + w.ml), a.part_o = reinterpret_cast<float *>(base + w.o);
  a.q_stride = q_stride, a.kv_stride = kv_stride;
  a.q_layer = q_stride * s->batch, a.kv_layer = k_new ? kv_stride * s->batch : 0;      // (several layers: okv8_decode_step, contiguous)
  a.codes_layer = codes_layer_bytes(c), a.scales_layer = scales_layer_floats(c), a.tails_layer = tails_layer_halves(c);
  a.scale_log2e = (float)(1.4426950408889634 / (c->head_dim == 128 ? 11.313708498984761 : 8.0));
  a.batch = s->batch, a.main_slots = w.slots, a.appends = s->appends, a.layers = layers, a.slot0 = 0;
  a.max_stretches = planned ? 0 : w.stretches;
  a.out = out, a.out_fp32 = c->out_dtype;
  if (const int waves = whole_waves(c, s->batch, layers)) {
    by_format<WholeLaunch8>(c, a, dim3((unsigned)(layers * s->batch * c->n_kv_heads)), waves, stream);
    return hip_result(who, hipGetLastError());
  }
  a.main_blocks = (w.stretches * c->n_kv_heads + 3) / 4;
  const int64_t blocks = (int64_t)layers * (a.main_blocks + (s->batch * c->n_kv_heads + 3) / 4);
  by_format<AttnLaunch8>(c, a, dim3((unsigned)blocks), streamed(c), stream);
  Merge8 m;
  m.plan = a.plan, m.part_o = a.part_o, m.part_ml = a.part_ml, m.out = out;
  m.batch = s->batch, m.H = c->n_q_heads, m.main_slots = w.slots, m.layers = layers, m.out_fp32 = c->out_dtype;
  const int64_t rows = (int64_t)layers * s->batch * c->n_q_heads;
  const bool wide = w.stretches >= 16 * s->batch;
  if (c->head_dim == 128) {
    if (wide) hipLaunchKernelGGL((merge8_kernel<128, 4>), dim3((unsigned)rows), dim3(256), 0, stream, m);
    else hipLaunchKernelGGL((merge8_kernel<128, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, m);
  } else {
    if (wide) hipLaunchKernelGGL((merge8_kernel<64, 4>), dim3((unsigned)rows), dim3(256), 0, stream, m);
    else hipLaunchKernelGGL((merge8_kernel<64, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, m);
  }
  return hip_result(who, hipGetLastError());
}

int begin(const char *who, const okv8_cache *c, const okv8_step *s, const Workspace8 &w) {
  hipLaunchKernelGGL(plan8_kernel, dim3(1), dim3(kPlanThreads), 0, static_cast<hipStream_t>(s->stream), s->seqs, s->lens, s->batch, s->appends,
                     cache_of(c, 0).s, w.stretches, plan_of(w, s->workspace));
  return hip_result(who, hipGetLastError());
}

}  // namespace

}  // namespace okv

using namespace okv;

extern "C" {

int64_t okv8_codes_bytes(const okv8_cache *c) {
  if (const char *why = shape_problem(c)) return report(OKV_EINVAL, "okv8_codes_bytes: %s", why);
  return codes_layer_bytes(c) * c->n_layers;
}
int64_t okv8_scales_bytes(const okv8_cache *c) {
  if (const char *why = shape_problem(c)) return report(OKV_EINVAL, "okv8_scales_bytes: %s", why);
  return scales_layer_floats(c) * c->n_layers * 4;
}
int64_t okv8_tails_bytes(const okv8_cache *c) {
  if (const char *why = shape_problem(c)) return report(OKV_EINVAL, "okv8_tails_bytes: %s", why);
  return tails_layer_halves(c) * c->n_layers * 2;
}
int64_t okv8_workspace_bytes(const okv8_cache *c, int32_t max_batch) {
  if (const char *why = shape_problem(c)) return report(OKV_EINVAL, "okv8_workspace_bytes: %s", why);
  if (max_batch < 1 || max_batch > OKV8_MAX_BATCH) return report(OKV_EINVAL, "okv8_workspace_bytes: batch must be in [1, %d]", OKV8_MAX_BATCH);
  // (a launch of several layers cuts the sequences less often: with few of them it may need less than one of a single layer)
  return std::max(workspace_of(c, max_batch, 1).bytes, workspace_of(c, max_batch, std::min(c->n_layers, kLayersAbreast)).bytes);
}

int okv8_store(const okv8_cache *c, int32_t layer, int32_t n_layers, int32_t batch, const int32_t *seqs, const int32_t *starts,
               const int32_t *lens, int64_t n_rows, const void *k, const void *v, int64_t row_stride, int64_t layer_stride, void *stream) {
  return rows_call("okv8_store", true, c, layer, n_layers, batch, seqs, starts, lens, n_rows, k, v, row_stride, layer_stride, stream);
}
int okv8_load(const okv8_cache *c, int32_t layer, int32_t n_layers, int32_t batch, const int32_t *seqs, const int32_t *starts,
              const int32_t *lens, int64_t n_rows, void *k, void *v, int64_t row_stride, int64_t layer_stride, void *stream) {
  return rows_call("okv8_load", false, c, layer, n_layers, batch, seqs, starts, lens, n_rows, k, v, row_stride, layer_stride, stream);
}

int okv8_step_begin(const okv8_cache *c, const okv8_step *s) {
  if (const int rc = step_problem("okv8_step_begin", c, s)) return rc;
  return begin("okv8_step_begin", c, s, workspace_of(c, s->batch, 1));
}

int okv8_decode_attn(const okv8_cache *c, const okv8_step *s, int32_t layer, const void *q, int64_t q_stride, const void *k_new,
                     const void *v_new, int64_t kv_stride, void *out) {
  if (const int rc = step_problem("okv8_decode_attn", c, s)) return rc;
  if (layer < 0 || layer >= c->n_layers) return report(OKV_EINVAL, "okv8_decode_attn: layer out of range");
  if (!q || !out || !aligned16(q) || !aligned16(out)) return report(OKV_EINVAL, "okv8_decode_attn: NULL or misaligned pointer");
  if ((k_new != nullptr) != (s->appends == 1) || (v_new != nullptr) != (s->appends == 1))
    return report(OKV_EINVAL, "okv8_decode_attn: k_new and v_new are given if, and only if, the step appends");
  if (!aligned16(k_new) || !aligned16(v_new)) return report(OKV_EINVAL, "okv8_decode_attn: misaligned pointer");
  if (q_stride < (int64_t)c->n_q_heads * c->head_dim || q_stride % 8 ||
      (s->appends && (kv_stride < (int64_t)c->n_kv_heads * c->head_dim || kv_stride % 8)))
    return report(OKV_EINVAL, "okv8_decode_attn: strides must be multiples of 8 and at least a row");
  return attend("okv8_decode_attn", c, s, workspace_of(c, s->batch, 1), true, layer, 1, q, q_stride, k_new, v_new, kv_stride, out);
}

int okv8_decode_step(const okv8_cache *c, const okv8_step *s, const void *q, const void *k_new, const void *v_new, void *out) {
  if (const int rc = step_problem("okv8_decode_step", c, s)) return rc;
  if (!q || !out || !aligned16(q) || !aligned16(out) || !aligned16(k_new) || !aligned16(v_new))
    return report(OKV_EINVAL, "okv8_decode_step: NULL or misaligned pointer");
  if ((k_new != nullptr) != (s->appends == 1) || (v_new != nullptr) != (s->appends == 1))
    return report(OKV_EINVAL, "okv8_decode_step: k_new and v_new are given if, and only if, the step appends");
  const Workspace8 w = workspace_for(c, s);
  const bool planned = s->batch > 64 && !whole_waves(c, s->batch, w.layers);
  int rc = planned ? begin("okv8_decode_step", c, s, w) : OKV_OK;
  const int64_t q_row = (int64_t)c->n_q_heads * c->head_dim, kv_row = (int64_t)c->n_kv_heads * c->head_dim;
  for (int32_t l = 0; rc == OKV_OK && l < c->n_layers; l += w.layers) {
    const auto at = [&](const void *p, int64_t row, int64_t size) { return p ? static_cast<const char *>(p) + l * s->batch * row * size : nullptr; };
    rc = attend("okv8_decode_step", c, s, w, planned, l, std::min(w.layers, c->n_layers - l), at(q, q_row, 2), q_row, at(k_new, kv_row, 2), at(v_new, kv_row, 2), kv_row,
                const_cast<char *>(at(out, q_row, c->out_dtype ? 4 : 2)));
  }
  return rc;
}

}  // extern "C"
