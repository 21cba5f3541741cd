// Several new tokens of a sequence at once over the fp16 cache (include/okv_chunk.h): appending with rotation, and attention of the rows, for gfx950.
//
// Appending moves 4 d (H + 2 G) bytes a row and is bound by HBM: 24 prompts of 100 to 2000 tokens, 32 / 8 heads x 128, 119 us (607 MB, 5.1 TB/s).
//
// Attention, out = sum_i softmax_i(s) v_i with the running maximum and sum of one pass.  Scores are the product K (rows: keys) x Q^T (columns: the rows of a KV head's queries, 32 of them in a
// wavefront): a lane then has 16 keys of one row, so the maximum and the sum take one exchange between halves of the wavefront, and the weights are where the second product, V^T x weights, wants
// them if its keys are taken in the order 4 h .. 4 h + 3, 8 + 4 h .. 11 + 4 h of every 16 (h the half).  V^T's operand comes from LDS by the load that transposes four rows of 16.
// Keys and values go from memory straight into LDS, two blocks ahead.  Many rows: bound by the matrix cores and the vector unit beside them (2.1 us a block of 64 keys and 128 rows, two workgroups to a
// compute unit: 1024 cycles of products and 850 of softmax for each wavefront); a chunk of 512 tokens behind some 58 000 keys 476 us, 1.00 PFLOP/s, 8 prompts of 2048 to 4096 (32 heads x 128) 901 us,
// 0.84 PFLOP/s.  Few rows: bound by HBM; 5 tokens for each of 32 sequences of up to 4096 keys, 32 / 8 heads x 128, 59 us (337 MB, 5.7 TB/s) and 5 to join.
// For an fp16 result weights are fp16 numbers in the second product; for fp32 two each (hi + lo), half as many products again.
#include "okv_chunk.h"
#include "okv_host.h"
#include "okv_lanes.h"
#include "okv_report.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "okv.h"

namespace okv {

namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));

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
    if (ended != ~(uint64_t)0) break;
  }
  return b < r.batch && r.starts[b] <= row ? b : -1;
}

constexpr int kAppendWaves = 4;

// Stores stay in the caches: past them (and loads too) 24 prompts of 100 to 2000 tokens take 109 us instead of 119, but the attention that comes next and reads what is new takes as much more (8 prompts of 2048
// behind as many, 32 / 8 heads x 128, both launches: 410 us either way; 16 of 300, 40 heads x 64: 72, past them 76 to 89).
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
  if (row < first || row >= last) return;                // (starts that do not ascend)
  const bool known = s >= 0 && s < c.max_seqs;
  if (known) len = max(r.lens[s], 0);
  const int token = len - (last - row);                  // (past the capacity: turned like others, and not stored)
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
  if (!known || token < 0 || token >= c.capacity || (c.refused && *c.refused)) return;
  const int32_t *table_row = c.table + (int64_t)s * c.width;
  // (a page that is none of the pool's: there is no place for the token, and another sequence's would lose its own)
  if (c.table && (unsigned)table_row[token >> 4 >> c.log2_tiles] >= (unsigned)c.n_blocks) return;
  const int64_t at = tile_at<D>(c, table_row, s, token >> 4) + (token & 15) * D;
  for (int g = slot; g < c.G; g += kHeads) {
    _Float16 *to = c.kv + at + head_offset<D>(c, g);
    move(a.k + row * a.kv_stride + g * D, to);
    const _Float16 *v = a.v + row * a.kv_stride + g * D;
    *reinterpret_cast<half8 *>(to + v_offset<D>(c) + 8 * unit) = *reinterpret_cast<const half8 *>(v + 8 * unit);
    *reinterpret_cast<half8 *>(to + v_offset<D>(c) + 8 * unit + D / 2) = *reinterpret_cast<const half8 *>(v + 8 * unit + D / 2);
  }
}

// ---- attention ------------------------------------------------------------------------------------

struct Plan;
struct Attend {
  const _Float16 *q;
  void *out;
  int64_t q_stride;
  float scale, cap;                      // of scores in units of log 2: scale log2(e), or with a cap 2 log2(e) scale / cap and cap log2(e)
  int32_t window;                        // 0: none
  int32_t may_cut;                       // whether keys may be cut among workgroups (a second launch joins them): 0, or the most items that the launch has workgroups for (see span_of)
  const float *slopes;
  const int32_t *prefix;
  Plan *plan;                            // in the workspace
  char *cuts;                            // in the workspace
  float *parts;                          // results of pieces of rows' keys: kRows x D sums, and behind them kRows maxima and kRows sums of weights
};

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kRaise = 8.f;            // the maximum is raised when a score is this far above it
// Weights are 2^(s - m + kLift): at most 2^15, and normal numbers in fp16 down to 2^-21 of the largest
constexpr float kLift = 7.f;
constexpr float kLowest = -3e38f;        // the maximum of no scores: finite, so that less it -infinity is that
constexpr float kNearCap = 64 * kLog2e;   // above it: see the tanh
constexpr int kRing = 2;                 // blocks of keys, and of values, in LDS

// Rows are the n R rows (tokens, and for each its R query heads) of a sequence and KV head; a wavefront has 32 of them, whose blocks of keys go by.
// Few rows: a workgroup has 32, each wavefront every fourth block of 32 keys, and joins them.  Many: a workgroup has 128, a wavefront 32, and all share blocks of 64 keys.
template <int D, bool FEW>
struct Form {
  static constexpr int kWaves = FEW && D == 128 ? 2 : 4, kThreads = 64 * kWaves;
  static constexpr int kRows = FEW ? 32 : 32 * kWaves, kKeys = FEW ? 32 : 64, kStep = FEW ? kWaves * kKeys : kKeys;      // keys of a step of the workgroup
  static constexpr int kBlockBytes = kKeys * D * 2, kLoads = kBlockBytes / 1024 / (FEW ? 1 : kWaves);                   // loads of a wavefront per block of keys (or values)
  static constexpr int kLds = (FEW ? kWaves : 1) * 2 * kRing * kBlockBytes;
  static constexpr int kPartFloats = kRows * (D + 2);
  // How keys are cut (see Plan): workgroups that run at a time, and in steps what a piece costs beside its own, what joining does, and what is never cut
  static constexpr int kSlots = 512, kUncut = 512 / kStep, kLeast = 256 / kStep;
  static constexpr float kPerPiece = FEW ? 1.f : 6.f, kPerJoin = FEW ? 3.f : 6.f;
  static constexpr int kPieces = 512;                   // that steps come to at most, where tiles are cut into equal pieces
  __host__ __device__ static int stretches(const int G) { return kSlots / G > 1 ? kSlots / G : 1; }
  __host__ __device__ static int64_t parts(const int G) { return 2 * (FEW ? (int64_t)stretches(G) * G : (int64_t)kPieces); }      // results of pieces
};

__device__ __forceinline__ half8 transposed(const char *first, const char *second) {
  typedef __attribute__((address_space(3))) short4v *at;
  const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)first), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)second);
  const half4 x = __builtin_bit_cast(half4, a), y = __builtin_bit_cast(half4, b);
  return half8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// What all lanes have the same, in scalar registers
__device__ __forceinline__ int uniform(const int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const char *uniform(const char *p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const char *>((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}
// One 16-byte-per-lane load from `base` + off straight into LDS: lane l's bytes land at lds + 16 l.  Written as assembly because the compiler, which cannot tell the block being
// written from the one being read, waits for all such loads in front of every LDS read otherwise.  m0 is left as it was found.
// ONCE: nobody else reads these bytes soon, past the caches (5 tokens for each of 32 sequences of up to 4096: 82 -> 76 us; with shared blocks 42 -> 45).
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const char *base, const uint32_t off, const uint32_t lds) {
  uint32_t found;
  if constexpr (ONCE)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3 nt\n\ts_mov_b32 m0, %0"
                 : "=&s"(found)
                 : "s"(uniform((int)lds)), "v"(off), "s"(uniform(base))
                 : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(found)
                 : "s"(uniform((int)lds)), "v"(off), "s"(uniform(base))
                 : "memory");
}
template <int N>
__device__ __forceinline__ void wait_for_loads() {      // until N are outstanding
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void barrier_leaving_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The steps of keys that some row of a tile sees, in order: `ahead` of the prefix, and those from `first` on
struct Keys {
  int ahead, first, total;
};
template <class F>
__device__ __forceinline__ Keys keys_of(const int n, const int base, const int len, const int prefix, const int window, const int R, const int tile) {
  const int pos0 = min(base + tile * F::kRows / R, len - 1), pos1 = min(base + min((tile * F::kRows + F::kRows - 1) / R, n - 1), len - 1);
  Keys k;
  k.first = window == 0 || pos0 < window ? 0 : (pos0 - window + 1) / F::kStep;
  k.ahead = min((prefix + F::kStep - 1) / F::kStep, k.first);
  k.total = k.ahead + max((max(pos1 + 1, prefix) + F::kStep - 1) / F::kStep - k.first, 0);
  return k;
}

// What workgroups do.  The rows of every sequence and KV head are cut into tiles (`tiles` of a sequence, each for G heads: its items), whose keys are walked in steps.  Where workgroups that take an item
// each would leave much of the chip idle, keys are cut among them, and a second launch joins the results.
//   many rows   every tile of a sequence is cut into as many pieces (`cuts`), of `span` steps at most
//   few rows    the steps of all tiles, one tile after the other, are shared out in stretches of `span`: G workgroups take a stretch, one for each head, which ends some tiles, holds some and
//               begins one.  (Heads side by side: their keys adjoin in memory.)
// Lengths are on the device: every wavefront finds this out for itself, a lane per sequence; beyond 64 sequences a launch of one workgroup adds up chunks of 64 first.
constexpr int kNone = 0x3fffffff;
struct Sequence {
  int first, n, s, len, prefix;          // its first row, its rows, its row of the table (below 0: there is none), its tokens (at most the capacity), those of its prefix
  int base;                              // the first row's position: rows past the capacity, which the pool has no tokens of, have the last token's
  int tiles, steps;                      // steps: of its last tile, which sees the most keys; others' are taken to be as many
};
struct Plan {                            // in the workspace, for more than 64 sequences; before each chunk of 64, and behind the last
  int span, unused;
  int pieces[OKV_CHUNK_MAX_BATCH / 64 + 1], cut_pieces[OKV_CHUNK_MAX_BATCH / 64 + 1], cut_tiles[OKV_CHUNK_MAX_BATCH / 64 + 1];
  uint64_t steps[OKV_CHUNK_MAX_BATCH / 64 + 1];      // of one head
};
constexpr int64_t kPlanBytes = 2048;
static_assert(sizeof(Plan) <= kPlanBytes, "");
// A tile that is cut, for the launch that joins its pieces, behind the plan: few rows, of the workgroup that takes its second piece; many, in order
struct Cut {
  int first, n, tile, g;                 // of its sequence: the first row, and rows
  int slot, slot1, apart, cuts;          // its pieces' results: slot, slot1, slot1 + apart, ..; cuts 0: there is none
};
constexpr int kMostCuts = 1024;
constexpr int64_t kCutBytes = 16 + kMostCuts * (int64_t)sizeof(Cut);      // (many rows: how many there are comes first)

template <class F>
__device__ __forceinline__ Sequence sequence_at(const Pool &c, const Rows &r, const Attend &a, const int b) {
  Sequence q{0, 0, -1, 0, 0, 0, 0, 0};
  if (b >= r.batch) return q;
  int last;
  rows_of(r, b, q.first, last);
  q.n = last - q.first;
  q.base = -q.n;
  const int s = r.seqs ? r.seqs[b] : b;
  if (s >= 0 && s < c.max_seqs) {
    q.s = s;
    const int lens = max(r.lens[s], 0);
    q.len = min(lens, c.capacity);
    q.base = min(lens - q.n, q.len);
    if (a.prefix) q.prefix = min(max(a.prefix[s], 0), q.len);
  }
  q.tiles = (int)(((int64_t)q.n * c.R + F::kRows - 1) / F::kRows);
  if (q.tiles) q.steps = max(keys_of<F>(q.n, q.base, q.len, q.prefix, a.window, c.R, q.tiles - 1).total, 1);      // (an item without keys is a step, too: its rows are 0)
  return q;
}
__device__ __forceinline__ int cuts_of(const Sequence &q, const int span) { return (int)(((unsigned)q.steps + (unsigned)span - 1) / (unsigned)span); }

// The span that is expected to take the least time, kNone: nothing is cut.  P pieces of up to s steps (W in all) on kSlots workgroups at a time, two to a compute unit, take s + kPerPiece where
// P <= kSlots, kAlone of that where each has a unit to itself, else (W + P kPerPiece) / kSlots and half a piece until the last one has ended; kPerJoin is added where any are cut.  us with kAlone .6 / 1: 8
// sequences of 32 tokens 31.0 / 34.6, 5 of 33 to 301 (40 heads x 64) 37.0 / 40.5, 16 of 1 to 600 behind 6000 338 / 330; with kPerPiece 4 and kPerJoin 10, 1000 rows of 8 heads 54.9 (38.5).
// sum(f) and most(f): over all sequences; pieces_at(s, work, items): how many with spans of s, a lane a span.
// Many rows: starts that do not ascend may come to more items than n_rows rows have; some pieces then have no workgroup, and what says where a cut tile's results are would not be written for the launch
// that joins them: nothing is cut.  (Few rows: as many workgroups as there are stretches, whatever the starts.)
constexpr float kAlone = .6f;
template <class F, bool FEW, class Sum, class Most, class PiecesAt>
__device__ __forceinline__ int span_of(const Pool &c, const Attend &a, const Sum &sum, const Most &most, const PiecesAt &pieces_at) {
  if (!a.may_cut) return kNone;
  const float work = sum([](const Sequence &q) { return (float)q.tiles * (float)q.steps; }) * c.G, items = sum([](const Sequence &q) { return (float)q.tiles; }) * c.G;
  const float longest = most([](const Sequence &q) { return (float)q.steps; });
  auto time = [&](const float pieces, const float s) {
    return pieces <= F::kSlots / 2 ? kAlone * (s + F::kPerPiece) : pieces <= F::kSlots ? s + F::kPerPiece : (work + pieces * F::kPerPiece) * (1.f / F::kSlots) + .5f * (s + F::kPerPiece);
  };
  const float best = time(items, longest);
  if constexpr (FEW) {
    const float stretches = (float)F::stretches(c.G), even = fmaxf(ceilf(work * 1.0001f / (stretches * c.G)), (float)F::kLeast);
    if (longest > F::kUncut && even + (items / (stretches * c.G) + 1.f) * F::kPerPiece + F::kPerJoin < best) return uniform((int)fminf(even, 1e9f));
    return kNone;
  } else {
    if (items > (float)a.may_cut || best < 1.2f * fmaxf(F::kPerJoin, work * (1.f / F::kSlots))) return kNone;      // (items of a launch are below 2^24: the sum is exact)
    // a lane a span: the longest item in 2 .. 49 pieces, and from a fourth to four times an even share
    const int lane = threadIdx.x & 63;
    const float least = fmaxf(1.f, ceilf(work * (1.0001f / F::kPieces)));
    const float s = fminf(fmaxf(ceilf(lane < 48 ? longest / (float)(lane + 2) : work * ((float)(lane - 47) * .25f / F::kSlots)), least), 1e9f);
    const float pieces = pieces_at(s, work, items);
    const float mine = time(pieces, fminf(longest, s)) + F::kPerJoin, shortest = -wave_max(-mine);
    if (!(shortest < best)) return kNone;
    return __builtin_amdgcn_readlane((int)s, __ffsll((unsigned long long)__ballot(mine == shortest)) - 1);
  }
}

__device__ __forceinline__ float about(const float s, const float work, const float items) { return fmaxf(items, work / s + .5f * items); }      // pieces, on the average

// The chunk of 64 sequences with the index-th of what `before` counts, a lane a sequence
template <class F, bool FEW>
struct Chunk {
  Sequence q;                            // this lane's
  int b0, span, at;                      // the chunk's first sequence; its number
  const Plan *plan;                      // NULL: the only chunk
  __device__ __forceinline__ Chunk(const Pool &c, const Rows &r, const Attend &a) : b0(0), at(0), plan(nullptr) {
    if (r.batch > 64) {
      plan = a.plan;
      span = uniform(plan->span);
      return;
    }
    q = sequence_at<F>(c, r, a, threadIdx.x & 63);
    span = span_of<F, FEW>(c, a, [&](const auto &f) { return wave_sum(f(q)); }, [&](const auto &f) { return wave_max(f(q)); }, [&](const float s, const float work, const float items) {
      if (r.batch > 16) return about(s, work, items);
      const float over = 1.f / s;
      float pieces = 0.f;
      for (int b = 0; b < r.batch; ++b) pieces += (float)lane_value(q.tiles, b) * ceilf((float)lane_value(q.steps, b) * over);
      return pieces * c.G;
    });
  }
  template <class T>
  __device__ __forceinline__ bool find(const Pool &c, const Rows &r, const Attend &a, const T (Plan::*before)[OKV_CHUNK_MAX_BATCH / 64 + 1], const T index) {
    if (!plan) return true;
    const int lane = threadIdx.x & 63, chunks = (r.batch + 63) / 64;
    at = __popcll(__ballot(lane < chunks && (plan->*before)[min(lane + 1, chunks)] <= index));
    if (at >= chunks) return false;
    b0 = 64 * at;
    q = sequence_at<F>(c, r, a, b0 + lane);
    return true;
  }
  __device__ __forceinline__ int cut_tiles(const Pool &c, const Rows &r) const {      // of all sequences (before find())
    if (plan) return plan->cut_tiles[(r.batch + 63) / 64];
    return lane_value(wave_scan(cuts_of(q, span) > 1 ? q.tiles * c.G : 0), 63);
  }
  template <class T>
  __device__ __forceinline__ T first(const T (Plan::*before)[OKV_CHUNK_MAX_BATCH / 64 + 1]) const { return plan ? (plan->*before)[at] : 0; }
};

struct Piece {
  Sequence q;
  int tile, g, begin, end;               // steps of its tile's q.steps
  int slot;                              // of its results in the workspace, below 0: it is whole
  int cuts, cut, cut_tile, apart;        // pieces of the tile, and which one this is; the number of the tile among those that are cut; slots from a piece to the next
};
__device__ __forceinline__ Sequence of_lane(const Sequence &q, const int lane) {
  return {lane_value(q.first, lane), lane_value(q.n, lane), lane_value(q.s, lane), lane_value(q.len, lane), lane_value(q.prefix, lane), lane_value(q.base, lane), lane_value(q.tiles, lane), lane_value(q.steps, lane)};
}
// Items of a sequence: the heads of a tile next to each other, so that those of a head are on the same XCD where they are a multiple of eight; tiles that see the most keys first
__device__ __forceinline__ void set_item(Piece &p, const Pool &c, const int item) {
  const int rank = uniform(item / c.G);
  p.g = item - rank * c.G;
  p.tile = p.q.tiles - 1 - rank;
}
// all part / parts, rounded down; in 32 bits where they suffice (a division of 64 is 150 instructions)
__device__ __forceinline__ int share(const int all, const int part, const int parts) {
  if (all == parts) return part;
  if (parts == 1) return part ? all : 0;
  if ((unsigned)all < 65536u && (unsigned)part < 65536u) return uniform((int)((unsigned)all * (unsigned)part / (unsigned)parts));
  return uniform((int)((uint64_t)(unsigned)all * (unsigned)part / (unsigned)parts));
}
// The index-th piece, where items are whole or cut into equal pieces.  A sequence's first cuts come first: tiles read the same keys together
template <class F, bool FEW>
__device__ __forceinline__ bool piece_of(Piece &p, Chunk<F, FEW> &k, const Pool &c, const Rows &r, const Attend &a, const int index) {
  if (!k.find(c, r, a, &Plan::pieces, index)) return false;
  const int cuts = cuts_of(k.q, k.span), mine = k.q.tiles * c.G * cuts, within_chunk = index - k.first(&Plan::pieces);
  const int upto = wave_scan(mine);
  const uint64_t ended = __ballot(upto <= within_chunk);
  if (ended == ~(uint64_t)0) return false;
  const int at = __popcll(ended);
  p.q = of_lane(k.q, at);
  p.cuts = lane_value(cuts, at);
  const int within = within_chunk - lane_value(upto - mine, at), items = p.q.tiles * c.G;
  if ((unsigned)within >= (unsigned)(items * p.cuts)) return false;      // (starts that do not ascend: sums past 2^31)
  const int cut = uniform(within / items);
  set_item(p, c, within - cut * items);
  p.begin = share(p.q.steps, cut, p.cuts), p.end = share(p.q.steps, cut + 1, p.cuts);
  p.slot = -1;
  if (p.cuts > 1) {
    const int cut_mine = cuts > 1 ? mine : 0, cut_upto = wave_scan(cut_mine);
    p.slot = k.first(&Plan::cut_pieces) + lane_value(cut_upto - cut_mine, at) + within;
    p.cut = cut, p.apart = items;
    const int tiles_mine = cuts > 1 ? k.q.tiles * c.G : 0, tiles_upto = wave_scan(tiles_mine);
    p.cut_tile = k.first(&Plan::cut_tiles) + lane_value(tiles_upto - tiles_mine, at) + within - cut * items;
  }
  return true;
}
// Where step `step` of all tiles' lies: its sequence (its number: b), the tile (its rank: those that see the most keys first) and the step of the tile
template <class F, bool FEW>
__device__ __forceinline__ bool step_of(Sequence &q, int &b, int &rank, int &within, Chunk<F, FEW> &k, const Pool &c, const Rows &r, const Attend &a, const uint64_t step) {
  if (!k.find(c, r, a, &Plan::steps, step)) return false;
  const uint64_t mine = (uint64_t)(unsigned)k.q.tiles * (unsigned)k.q.steps, within_chunk = step - k.first(&Plan::steps);
  const uint64_t upto = wave_scan(mine);
  const uint64_t ended = __ballot(upto <= within_chunk);
  if (ended == ~(uint64_t)0) return false;
  const int at = __popcll(ended);
  const uint64_t rest = within_chunk - lane_value(upto - mine, at);
  q = of_lane(k.q, at);
  b = k.b0 + at;
  rank = uniform((int)(rest / (unsigned)q.steps));
  within = uniform((int)(rest - (uint64_t)(unsigned)rank * (unsigned)q.steps));
  return true;
}

// One workgroup: what more than 64 sequences come to
constexpr int kPlanThreads = 1024, kPlanEach = OKV_CHUNK_MAX_BATCH / kPlanThreads;
template <class F, bool FEW>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(Pool c, Rows r, Attend a) {
  constexpr int kPlanWaves = kPlanThreads / 64;
  __shared__ float shared[kPlanWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunks = (r.batch + 63) / 64;
  Sequence q[kPlanEach];
#pragma unroll
  for (int i = 0; i < kPlanEach; ++i) q[i] = sequence_at<F>(c, r, a, i * kPlanThreads + (int)threadIdx.x);
  auto all = [&](float x, const bool largest) {
    x = largest ? wave_max(x) : wave_sum(x);
    __syncthreads();
    if (lane == 0) shared[wave] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) x = largest ? fmaxf(x, shared[w]) : x + shared[w];
    return x;
  };
  auto each = [&](const auto &f, const bool largest) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < kPlanEach; ++i) x = largest ? fmaxf(x, f(q[i])) : x + f(q[i]);
    return all(x, largest);
  };
  const int span = span_of<F, FEW>(c, a, [&](const auto &f) { return each(f, false); }, [&](const auto &f) { return each(f, true); }, about);
  Plan &plan = *a.plan;
#pragma unroll
  for (int i = 0; i < kPlanEach; ++i) {                  // chunk 16 i + wave
    const int cuts = cuts_of(q[i], span), items = q[i].tiles * c.G, chunk = i * kPlanWaves + wave;
    const int pieces = wave_scan(items * cuts), cut_pieces = wave_scan(cuts > 1 ? items * cuts : 0), cut_tiles = wave_scan(cuts > 1 ? items : 0);
    const uint64_t steps = wave_scan((uint64_t)(unsigned)q[i].tiles * (unsigned)q[i].steps);
    if (lane == 63 && chunk < chunks) plan.pieces[chunk + 1] = pieces, plan.cut_pieces[chunk + 1] = cut_pieces, plan.cut_tiles[chunk + 1] = cut_tiles, plan.steps[chunk + 1] = steps;
  }
  __threadfence_block();
  __syncthreads();
  if (wave) return;
  const bool there = lane < chunks;
  const int pieces = wave_scan(there ? plan.pieces[lane + 1] : 0), cut_pieces = wave_scan(there ? plan.cut_pieces[lane + 1] : 0), cut_tiles = wave_scan(there ? plan.cut_tiles[lane + 1] : 0);
  const uint64_t steps = wave_scan(there ? plan.steps[lane + 1] : (uint64_t)0);
  if (there) plan.pieces[lane + 1] = pieces, plan.cut_pieces[lane + 1] = cut_pieces, plan.cut_tiles[lane + 1] = cut_tiles, plan.steps[lane + 1] = steps;
  if (lane == 0) plan.span = span, plan.pieces[0] = plan.cut_pieces[0] = plan.cut_tiles[0] = 0, plan.steps[0] = 0;
}

// The steps of a piece in which a wavefront has taken out values that are not finite, of those that not every row sees: none, or the first and the last
struct Odd {
  int first, last;
};

// `meanwhile` is called while the first blocks are on their way
template <int D, bool FEW, bool WIDE, bool SHAPED, class Meanwhile>
__device__ __forceinline__ void attend_piece(const Pool &c, const Attend &a, const Piece &piece, char *const lds, Odd &shared_odd, const Meanwhile &meanwhile) {
  using F = Form<D, FEW>;
  constexpr int kWaves = F::kWaves, kLoads = F::kLoads, kKeys = F::kKeys, kRowBytes = 2 * D, kParts = kKeys / 32;
  const Sequence &p = piece.q;
  // Few rows: each wavefront's own, in registers.  Many: everybody's, in LDS, set before the barrier that comes before the first step
  Odd odd{INT_MAX, -1};
  if (!FEW && threadIdx.x == 0) shared_odd = odd;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int row0 = piece.tile * F::kRows + (FEW ? 0 : wave * 32), row = row0 + col;         // of the sequence's n R rows
  const int token = row / c.R, head = piece.g * c.R + row - token * c.R;
  auto position = [&](const int token) { return min(p.base + token, p.len - 1); };
  const int pos = position(token);
  auto first_seen = [&](const int pos) { return a.window == 0 || pos < a.window ? 0 : pos - a.window + 1; };      // (but for the prefix)
  const int from = first_seen(pos);
  // of this wavefront's rows, and of the tile's
  const int token0 = uniform(row0 / c.R), token1 = min(uniform((row0 + 31) / c.R), p.n - 1);
  const bool idle = token0 >= p.n;
  const int pos0 = position(token0), pos1 = position(token1), from0 = first_seen(pos0), from1 = first_seen(pos1);
  const int tile_pos0 = position(uniform(piece.tile * F::kRows / c.R)), tile_pos1 = position(min(uniform((piece.tile * F::kRows + F::kRows - 1) / c.R), p.n - 1));
  const int tile_from1 = first_seen(tile_pos1);
  auto all_see = [&](const int key0) { return (key0 + kKeys - 1 <= tile_pos0 && key0 >= tile_from1) || key0 + kKeys <= p.prefix; };      // rows of the tile
  auto in_sight = [&](const int key0) { return !idle && ((key0 <= pos1 && key0 + kKeys > from0) || key0 < p.prefix); };                  // of some row of the wavefront

  // this piece's steps of the tile's
  Keys keys = keys_of<F>(p.n, p.base, p.len, p.prefix, a.window, c.R, piece.tile);
  keys.ahead = uniform(keys.ahead), keys.first = uniform(keys.first), keys.total = uniform(keys.total);
  const bool whole_tile = piece.slot < 0;
  const int i0 = whole_tile ? 0 : share(keys.total, piece.begin, p.steps), total = whole_tile ? keys.total : share(keys.total, piece.end, p.steps) - i0;
  auto key_at_step = [&](const int i) {                // this wavefront's first key of a step; past the end: the last again
    const int j = i0 + min(i, total - 1);
    return (j < keys.ahead ? j : keys.first + j - keys.ahead) * F::kStep + (FEW ? wave * kKeys : 0);
  };

  half8 qf[D / 16];
  {
    const _Float16 *q = a.q + (p.first + min(token, p.n - 1)) * a.q_stride + head * D + 8 * half;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) qf[k] = *reinterpret_cast<const half8 *>(q + 16 * k);
  }
  const float slope = SHAPED && a.slopes ? a.slopes[head] * kLog2e : 0.f;

  // Loads.  Row r of a block has its 16-byte pieces in units (D / 8) r .. of LDS, piece k in unit (D / 8) r + (k ^ turn(r)), turn 4 (r & 3) + ((r >> 2) & 3) (D = 64: of r / 2, one bit each):
  // sixteen rows' same piece, and the four pieces of 32 elements of four rows, are in different banks.  A load brings 1 KiB, 512 / D rows of a tile of 16.  FEW: a
  // wavefront has rings of its own and loads all of its blocks; else load j of a block is wavefront j % 4's.
  constexpr int kTileLoads = 16 * kRowBytes / 1024, kUnits = D / 8, kBases = FEW ? kLoads / kTileLoads : kLoads;
  static_assert(FEW || kWaves % kTileLoads == 0, "a wavefront's loads of a shared block are of the same rows of their tiles");
  const int lane_row = lane / kUnits;
  const uint32_t lane_base = lane_row * kRowBytes + 16 * ((lane % kUnits) ^ (D == 128 ? 4 * lane_row : 4 * ((lane_row >> 1) & 1) | (lane_row >> 2)));
  auto lane_offset = [&](const int j) { return (lane_base ^ (j * (D == 128 ? 16 : 32))) + j * 1024; };         // of load j of a tile
  const uint32_t shared_offset = lane_offset(wave % kTileLoads);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + (FEW ? wave * (F::kLds / kWaves) : 0);
  char *const mine = lds + (FEW ? wave * (F::kLds / kWaves) : 0);
  const int32_t *table_row = c.table + (int64_t)max(p.s, 0) * c.width;
  const char *pool = uniform(reinterpret_cast<const char *>(c.kv + head_offset<D>(c, piece.g)));
  const int64_t slab = (int64_t)2 * c.G * D << (4 + c.st_log2);
  const int last_tile = (p.len - 1) >> 4;
  int held_from = INT_MIN / 2, held = p.s;              // lane l: the block in entry held_from + l of the sequence's row of the table
  const char *bases[kBases];             // of the keys that were loaded last
  auto load = [&](const uint32_t more, const int slot) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      if constexpr (FEW) load_to_lds<true>(bases[j / kTileLoads] + more, lane_offset(j % kTileLoads), lds0 + slot * F::kBlockBytes + j * 1024);
      else load_to_lds<false>(bases[j] + more, shared_offset, lds0 + slot * F::kBlockBytes + (j * kWaves + wave) * 1024);
  };
  auto load_keys = [&](const int i, const int slot) {
    const int t0 = uniform(key_at_step(i)) / 16 + (FEW ? 0 : wave / kTileLoads);
#pragma unroll
    for (int j = 0; j < kBases; ++j) {
      const int t = min(t0 + (FEW ? j : j * (kWaves / kTileLoads)), last_tile), e = t >> c.log2_tiles, tb = t & ((1 << c.log2_tiles) - 1);
      if (c.table && (unsigned)(e - held_from) >= 64u) {
        held_from = e;
        held = min(max(table_row[min(e + lane, c.width - 1)], 0), c.n_blocks - 1);
      }
      const int block = __builtin_amdgcn_readlane(held, c.table ? e - held_from : 0);
      bases[j] = uniform(pool + 2 * (block * c.block_elems + (tb >> c.st_log2) * slab + (int64_t)(tb & ((1 << c.st_log2) - 1)) * (c.gg * 16 * D)));
    }
    load(0, slot);
  };
  const uint32_t behind = 2 * v_offset<D>(c);
  auto load_values = [&](const int slot) { load(behind, kRing + slot); };      // of the keys that were loaded last

  // where this lane's operands begin in a block; xor 32 k (keys' k-th 16 elements) or 64 e (values' e-th 32 elements)
  const int x4 = (lane >> 2) & 3, p4 = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
  uint32_t key_at, value_at0, value_at1;
  if constexpr (D == 128) {
    key_at = col * kRowBytes + 16 * (half ^ (4 * (col & 3) | ((col >> 2) & 3)));
    value_at0 = (4 * half + x4) * kRowBytes + 16 * (p4 ^ (4 * x4 | half)) + 8 * (lane & 1);
    value_at1 = (8 + 4 * half + x4) * kRowBytes + 16 * (p4 ^ (4 * x4 | (half + 2))) + 8 * (lane & 1);
  } else {
    key_at = col * kRowBytes + 16 * (half ^ (4 * ((col >> 1) & 1) | ((col >> 2) & 3)));
    value_at0 = (4 * half + x4) * kRowBytes + 16 * (p4 ^ (4 * (x4 >> 1) | half)) + 8 * (lane & 1);
    value_at1 = (8 + 4 * half + x4) * kRowBytes + 16 * (p4 ^ (4 * (x4 >> 1) | (half + 2))) + 8 * (lane & 1);
  }

  floatx16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = floatx16{};
  float m = kLowest, l = 0.f;
  // scores: keys 32 b + 8 (i / 4) + 4 half + i % 4 of this lane's row
  auto score = [&](floatx16 (&x)[kParts], const int slot) {
    const char *k0 = mine + slot * F::kBlockBytes;
#pragma unroll
    for (int b = 0; b < kParts; ++b) {
      x[b] = floatx16{};
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
        x[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8 *>(k0 + (key_at ^ (32 * k)) + b * 32 * kRowBytes), qf[k], x[b], 0, 0, 0);
    }
  };

  // A number that is not finite may be of a key that some row does not see, and 0 times it is not 0: it is taken out, and added at the end where it is seen
  auto take_out = [&](const int i, char *const v0) {
    bool found = false;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      u32x4 *at = reinterpret_cast<u32x4 *>(v0 + (FEW ? j : j * kWaves + wave) * 1024 + 16 * lane), w = *at;
      uint32_t any = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t bad = ((w[k] & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
        w[k] &= ~(bad - (bad >> 15));
        any |= bad;
      }
      if (any) {
        *at = w;
        found = true;
      }
    }
    if constexpr (FEW) {
      if (__ballot(found)) odd.first = min(odd.first, i), odd.last = i;
    } else if (found) {
      atomicMin(&shared_odd.first, i), atomicMax(&shared_odd.last, i);
    }
  };
  auto step = [&](auto last, const int i, const int slot, floatx16 (&x)[kParts], floatx16 (&next)[kParts]) {
    constexpr bool kLast = decltype(last)::value;
    wait_for_loads<0>();
    if constexpr (!FEW) barrier_leaving_loads();         // the next block of keys and this one of values are there, those before free
    if constexpr (!kLast) {
      load_values(slot ^ 1);
      if (!FEW || i + 2 < total) load_keys(i + 2, slot);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int key0 = uniform(key_at_step(i));
    char *const v0 = mine + (kRing + slot) * F::kBlockBytes;
    if (!all_see(key0)) {
      take_out(i, v0);
      if constexpr (!FEW) __syncthreads();
    }
    if (!in_sight(key0)) {
      if constexpr (!kLast)
        if ((FEW || i + 1 < total) && in_sight(uniform(key_at_step(i + 1)))) score(next, slot ^ 1);
      return;
    }
    const bool whole = (key0 + kKeys - 1 <= pos0 && key0 >= from1) || key0 + kKeys <= p.prefix;
    const int apart = pos - key0 - 4 * half;             // from the lane's first key to its row
    float by = a.scale, shift = 0.f;                     // scores in units of log 2 are by x + shift
    if constexpr (SHAPED) {
      // tanh(y) = 1 - 2 / (e^2y + 1) is off by 3 2^-24 of 1, whatever y: of a cap that is far above the scores more than they bear.  There (kNearCap) small y take their series, up to y^9: off by 2^-26 of itself
      // below 1/4, and by 12 2^-24 above.  us of 4 times 700 to
      // 1024 rows behind up to 8000 tokens, 16 / 8 heads x 128, cap 50: 170, with both for every cap 227
      if (a.cap > kNearCap) {
#pragma unroll
        for (int b = 0; b < kParts; ++b)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float z = x[b][j] * a.scale, y = z * (.5f / kLog2e), yy = y * y;
            const float series = fmaf(fmaf(fmaf(fmaf(62.f / 2835, yy, -17.f / 315), yy, 2.f / 15), yy, -1.f / 3) * yy, y, y);
            const float far = fmaf(2.f, __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(z)), 1.f);
            x[b][j] = fabsf(y) < .25f ? series : far;
          }
        by = a.cap;
      } else if (a.cap != 0.f) {
#pragma unroll
        for (int b = 0; b < kParts; ++b)
#pragma unroll
          for (int j = 0; j < 16; ++j) x[b][j] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(x[b][j] * a.scale));
        by = 2.f * a.cap, shift = a.cap;
      }
      if (a.slopes) {
        const float far = (float)apart;
        if (key0 + kKeys - 1 <= pos0) {                  // all keys before all rows: the distance is a difference
          const float nearest = fmaf(-slope, far, shift);
#pragma unroll
          for (int b = 0; b < kParts; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) x[b][j] = fmaf(x[b][j], by, fmaf(slope, (float)(32 * b + 8 * (j / 4) + j % 4), nearest));
        } else {
#pragma unroll
          for (int b = 0; b < kParts; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) x[b][j] = fmaf(-slope, fabsf(far - (float)(32 * b + 8 * (j / 4) + j % 4)), fmaf(x[b][j], by, shift));
        }
        by = 1.f, shift = 0.f;
      }
    }
    if (!whole) {
      const int fixed = p.prefix - key0 - 4 * half, upto = max(apart, fixed - 1), below = from - key0 - 4 * half;
#pragma unroll
      for (int b = 0; b < kParts; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int key = 32 * b + 8 * (j / 4) + j % 4;
          const bool hidden = (key > upto) | ((key < below) & (key >= fixed));
          x[b][j] = hidden ? -INFINITY : x[b][j];
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int b = 0; b < kParts; ++b)
#pragma unroll
      for (int j = 0; j < 16; j += 2) top = fmaxf(fmaxf(top, x[b][j]), x[b][j + 1]);
    top = fmaf(max_with_lane_xor<32>(top), by, shift);
    if (__ballot(top > m + kRaise)) {
      const float to = top > m + kRaise ? top : m, scale = __builtin_amdgcn_exp2f(m - to);
      l *= scale;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) o[e] *= scale;
      m = to;
    }
    __builtin_amdgcn_s_setprio(1);
    // The next block's scores under this one's weights (out of sight, or past the end of shared blocks: for nothing)
    if constexpr (!kLast) score(next, slot ^ 1);
    half8 hi[2 * kParts], lo[WIDE ? 2 * kParts : 1];
    const float less = kLift - m + shift;
    float sums[4] = {};
#pragma unroll
    for (int b = 0; b < kParts; ++b)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float w = __builtin_amdgcn_exp2f(fmaf(x[b][j], by, less));
        sums[j % 4] += w;
        hi[2 * b + j / 8][j % 8] = (_Float16)w;
        if constexpr (WIDE) lo[2 * b + j / 8][j % 8] = (_Float16)(w - (float)(_Float16)w);
      }
    l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
    // results: elements 32 e + 8 (i / 4) + 4 half + i % 4 of this lane's row
#pragma unroll
    for (int t = 0; t < 2 * kParts; ++t)
#pragma unroll
      for (int e = 0; e < D / 32; ++e) {
        const half8 vf = transposed(v0 + (value_at0 ^ (64 * e)) + t * 16 * kRowBytes, v0 + (value_at1 ^ (64 * e)) + t * 16 * kRowBytes);
        o[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, hi[t], o[e], 0, 0, 0);
        if constexpr (WIDE) o[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, lo[t], o[e], 0, 0, 0);
      }
    if constexpr (!FEW && !kLast) {
      // The order of what comes before, as far as operands allow: keys read eight operands ahead, two products of scores with 6 (D = 64: 12) other instructions and 2 (5) exponentials beside them, one of results with 4 and
      // 1.  us of 8 prompts of 2048 to 4096 (32 heads x 128) / a chunk of 512 behind some 58 000 keys: 928 / 478, with four products in a row 936 / 505, fewer instructions beside them
      // 1005 / 530, left to the compiler 965 / 500; without the priority that the products' wavefront has over the other one of its SIMD 957 / 504, with neither 980 / 518
      constexpr int kScores = kParts * D / 16, kResults = 2 * kParts * (D / 32) * (WIDE ? 2 : 1);
      __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);      // reads of LDS; 8: products, 2: other vector instructions, 0x400: exponentials
#pragma unroll
      for (int k = 0; k < kScores / 2; ++k) {
        __builtin_amdgcn_sched_group_barrier(8, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(2, 100 / kScores, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 40 / kScores, 0);
      }
#pragma unroll
      for (int k = 0; k < kResults; ++k) {
        __builtin_amdgcn_sched_group_barrier(8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(2, 4, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if (total == 0) meanwhile();
  if (total > 0) {
    load_keys(0, 0);
    floatx16 x[kParts], y[kParts];
    load_values(0);
    load_keys(1, 1);
    __builtin_amdgcn_sched_barrier(0);
    meanwhile();
    wait_for_loads<2 * kLoads>();
    if constexpr (!FEW) {
      __builtin_amdgcn_s_waitcnt(0xc07f);                // (what thread 0 has set is in LDS)
      barrier_leaving_loads();
    }
    if (in_sight(uniform(key_at_step(0)))) score(x, 0);
    // The last step has code of its own, brings nothing and computes no scores after its own: us of 4 sequences of 1 to 5 rows 8.07 -> 7.65, of 5 rows for each of 32 70.6 -> 67.5.  With shared blocks that
    // needs more registers than there are (872 after 876 for 8 prompts, but 181 after 170 with a cap); loads under a condition in every step take 965 after 909
    if constexpr (FEW) {
      int i = 0;
      for (; i + 2 < total; i += 2) {
        step(std::false_type{}, i, 0, x, y);
        step(std::false_type{}, i + 1, 1, y, x);
      }
      if (i + 1 < total) {
        step(std::false_type{}, i, 0, x, y);
        step(std::true_type{}, i + 1, 1, y, x);
      } else {
        step(std::true_type{}, i, 0, x, y);
      }
    } else {
      for (int i = 0;; i += 2) {
        step(std::false_type{}, i, 0, x, y);
        if (i + 1 >= total) break;
        step(std::false_type{}, i + 1, 1, y, x);
        if (i + 2 >= total) break;
      }
    }
    wait_for_loads<0>();                                 // nothing may still be on its way into LDS
    __syncthreads();
    if constexpr (!FEW) odd = {uniform(shared_odd.first), uniform(shared_odd.last)};
#pragma unroll 1
    for (int i = odd.first; i <= odd.last; ++i) {
      const int key0 = uniform(key_at_step(i));
      if (all_see(key0)) continue;
#pragma unroll 1
      for (int key = key0; key < min(key0 + kKeys, p.len); ++key) {
        const bool seen = (key <= pos && key >= from) || key < p.prefix;
        const _Float16 *v = c.kv + tile_at<D>(c, table_row, p.s, key >> 4) + head_offset<D>(c, piece.g) + v_offset<D>(c) + (key & 15) * D + 4 * half;
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const half4 w = *reinterpret_cast<const half4 *>(v + 32 * e + 8 * j);
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (seen && !(fabsf((float)w[q]) < INFINITY)) o[e][4 * j + q] += (float)w[q];
          }
      }
    }
  }
  l = sum_with_lane_xor<32>(l);
  float *parts = a.parts + (int64_t)max(piece.slot, 0) * F::kPartFloats;
  if constexpr (!FEW) {
    const int of_tile = wave * 32 + col;
    const float over = !whole_tile ? 1.f : l == 0.f ? 0.f : 1.f / l;
    if (!WIDE && whole_tile) {
      // Whole rows through LDS (each wavefront's in a place of its own), 16 bytes a lane
      constexpr int kStride = kRowBytes + 16;
      char *const own = lds + wave * (32 * kStride);
      static_assert(kWaves * 32 * kStride <= F::kLds, "");
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          half4 y;
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = (_Float16)(o[e][4 * i + j] * over);
          *reinterpret_cast<half4 *>(own + col * kStride + 64 * e + 16 * i + 8 * half) = y;
        }
#pragma unroll
      for (int k = 0; k < 32; k += 64 / kUnits) {
        const int r0 = row0 + k + lane_row, their_token = r0 / c.R;
        const u32x4 y = *reinterpret_cast<const u32x4 *>(own + (k + lane_row) * kStride + 16 * (lane % kUnits));
        if (their_token < p.n)
          *reinterpret_cast<u32x4 *>(static_cast<_Float16 *>(a.out) + ((int64_t)(p.first + their_token) * (c.G * c.R) + piece.g * c.R + r0 - their_token * c.R) * D + 8 * (lane % kUnits)) = y;
      }
      return;
    }
    if (token >= p.n) return;
    const int64_t to = !whole_tile ? of_tile * D : ((int64_t)(p.first + token) * (c.G * c.R) + head) * D;
    if (!whole_tile && half == 0) parts[F::kRows * D + of_tile] = m, parts[F::kRows * (D + 1) + of_tile] = l;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        floatx4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = o[e][4 * i + j] * over;
        *reinterpret_cast<floatx4 *>((!whole_tile ? parts : static_cast<float *>(a.out)) + to + 32 * e + 8 * i + 4 * half) = y;
      }
  } else {
    // The wavefronts' results through LDS (each has written to rings of its own only): a row's D sums, then the maxima and the sums of weights
    constexpr int kStride = D + 4, kEach = F::kLds / kWaves / 4;
    static_assert(32 * kStride + 64 <= kEach, "a wavefront's results fit its rings");
    float *const all = reinterpret_cast<float *>(lds), *const own = all + wave * kEach;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<floatx4 *>(own + col * kStride + 32 * e + 8 * i + 4 * half) = floatx4{o[e][4 * i], o[e][4 * i + 1], o[e][4 * i + 2], o[e][4 * i + 3]};
    if (half == 0) own[32 * kStride + col] = m, own[32 * kStride + 32 + col] = l;
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < 32 / kWaves; k += 8) {
    const int of_tile = wave * (32 / kWaves) + k + lane / 8, joined_row = piece.tile * 32 + of_tile, joined_token = joined_row / c.R;
    if (joined_token >= p.n) return;
    float most = kLowest, sum = 0.f, factor[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, all[w * kEach + 32 * kStride + of_tile]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      factor[w] = __builtin_amdgcn_exp2f(all[w * kEach + 32 * kStride + of_tile] - most);
      sum += all[w * kEach + 32 * kStride + 32 + of_tile] * factor[w];
    }
    const float over = !whole_tile ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
    const int64_t to = !whole_tile ? of_tile * D : ((int64_t)(p.first + joined_token) * (c.G * c.R) + piece.g * c.R + joined_row - joined_token * c.R) * D;
    if (!whole_tile && lane % 8 == 0) parts[F::kRows * D + of_tile] = most, parts[F::kRows * (D + 1) + of_tile] = sum;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      floatx4 y = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) y += *reinterpret_cast<const floatx4 *>(all + w * kEach + of_tile * kStride + 32 * e + 4 * (lane % 8)) * factor[w];
      y *= over;
      const int64_t at = to + 32 * e + 4 * (lane % 8);
      if (!whole_tile) *reinterpret_cast<floatx4 *>(parts + at) = y;
      else if constexpr (WIDE) *reinterpret_cast<floatx4 *>(static_cast<float *>(a.out) + at) = y;
      else *reinterpret_cast<half4 *>(static_cast<_Float16 *>(a.out) + at) = half4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
    }
    }
  }
}

template <int D, bool FEW, bool WIDE, bool SHAPED>
__global__ void __launch_bounds__((Form<D, FEW>::kThreads)) __attribute__((amdgpu_waves_per_eu(FEW && D == 128 ? 1 : 2, 2))) chunk_kernel(Pool c, Rows r, Attend a) {
  using F = Form<D, FEW>;
  __shared__ __attribute__((aligned(1024))) char lds[F::kLds];
  __shared__ Odd shared_odd;
  Chunk<F, FEW> k(c, r, a);
  Piece p;
  Cut *const cut = reinterpret_cast<Cut *>(a.cuts + 16);
  if (!FEW || k.span == kNone) {
    if constexpr (FEW) {
      if (a.may_cut && (int)blockIdx.x < F::stretches(c.G) * c.G && threadIdx.x == 0) cut[blockIdx.x].cuts = 0;
    } else if (a.may_cut && blockIdx.x == 0) {
      const int all = k.cut_tiles(c, r);
      if (threadIdx.x == 0) *reinterpret_cast<int *>(a.cuts) = all;
    }
    if (!piece_of(p, k, c, r, a, (int)blockIdx.x)) return;
    if (!FEW && p.slot >= 0 && p.cut == 0 && threadIdx.x == 0) cut[p.cut_tile] = {p.q.first, p.q.n, p.tile, p.g, p.slot, p.slot + p.apart, p.apart, p.cuts};
    attend_piece<D, FEW, WIDE, SHAPED>(c, a, p, lds, shared_odd, [] {});
    return;
  }
  if constexpr (FEW) {
    const int stretch = uniform((int)blockIdx.x / c.G), g = (int)blockIdx.x - stretch * c.G;
    if (stretch >= F::stretches(c.G)) return;
    int b, rank;
    const bool there = step_of(p.q, b, rank, p.begin, k, c, r, a, (uint64_t)(unsigned)stretch * (unsigned)k.span);
    p.g = g;
    if (threadIdx.x == 0) {                              // (the first stretch that begins in a tile says so)
      Cut one{};
      if (there && p.begin > 0 && p.begin <= k.span)
        one = {p.q.first, p.q.n, p.q.tiles - 1 - rank, g, (2 * stretch - 1) * c.G + g, 2 * stretch * c.G + g, 2 * c.G, 1 + (p.q.steps - p.begin + k.span - 1) / k.span};
      cut[blockIdx.x] = one;
    }
    if (!there) return;
    for (int left = k.span;;) {
      p.tile = p.q.tiles - 1 - rank;
      p.end = min(p.q.steps, p.begin + left);
      p.slot = p.begin > 0 ? 2 * stretch * c.G + g : p.end < p.q.steps ? (2 * stretch + 1) * c.G + g : -1;
      left -= p.end - p.begin;
      Sequence next = p.q;
      bool more = left > 0;
      auto look_ahead = [&] {
        if (!more || ++rank < p.q.tiles) return;
        rank = 0;
        do {
          if (!(more = ++b < r.batch)) return;
          next = of_lane(sequence_at<F>(c, r, a, b), 0);
        } while (next.tiles == 0);
      };
      attend_piece<D, FEW, WIDE, SHAPED>(c, a, p, lds, shared_odd, look_ahead);
      if (!more) return;
      p.q = next, p.begin = 0;
      __syncthreads();                                   // LDS is free again
    }
  }
}

// Joins the results of a tile's pieces, a workgroup for some rows
constexpr int kJoinThreads = 256;
template <int D>
constexpr int kJoinLanes = D / 4;                        // of a row, four elements each
template <int D>
constexpr int kJoinRows = kJoinThreads / kJoinLanes<D>;

template <int D, bool FEW, bool WIDE>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(Pool c, Attend a) {
  using F = Form<D, FEW>;
  constexpr int kLanes = kJoinLanes<D>;
  const int index = blockIdx.x / (F::kRows / kJoinRows<D>), lane = threadIdx.x % kLanes;
  if (!FEW && index >= *reinterpret_cast<const int *>(a.cuts)) return;
  const Cut t = reinterpret_cast<const Cut *>(a.cuts + 16)[index];
  const int of_tile = blockIdx.x % (F::kRows / kJoinRows<D>) * kJoinRows<D> + threadIdx.x / kLanes, row = t.tile * F::kRows + of_tile, token = row / c.R, head = t.g * c.R + row - token * c.R;
  if (t.cuts == 0 || token >= t.n) return;
  auto part = [&](const int cut) { return a.parts + (int64_t)(cut ? t.slot1 + (cut - 1) * t.apart : t.slot) * F::kPartFloats; };
  float m = kLowest, l = 0.f;
  for (int cut = lane; cut < t.cuts; cut += kLanes) m = fmaxf(m, part(cut)[F::kRows * D + of_tile]);
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  floatx4 o = {};
  for (int cut0 = 0; cut0 < t.cuts; cut0 += kLanes) {
    float factor = 0.f;
    if (cut0 + lane < t.cuts) {
      const float *one = part(cut0 + lane);
      factor = __builtin_amdgcn_exp2f(one[F::kRows * D + of_tile] - m);
      l += one[F::kRows * (D + 1) + of_tile] * factor;
    }
    for (int j0 = 0; j0 < min(kLanes, t.cuts - cut0); j0 += 8) {      // (past the last: that one again, for nothing)
      floatx4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const floatx4 *>(part(min(cut0 + j0 + j, t.cuts - 1)) + of_tile * D + 4 * lane);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (0 times a piece far below the largest counts, too: it makes a number that is not finite NaN)
        const float by = __shfl(factor, j0 + j, kLanes);
        if (cut0 + j0 + j < t.cuts) o += v[j] * by;
      }
    }
  }
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) l += __shfl_xor(l, o);
  o *= l == 0.f ? 0.f : 1.f / l;
  const int64_t at = ((int64_t)(t.first + token) * (c.G * c.R) + head) * D + 4 * lane;
  if constexpr (WIDE) *reinterpret_cast<floatx4 *>(static_cast<float *>(a.out) + at) = o;
  else *reinterpret_cast<half4 *>(static_cast<_Float16 *>(a.out) + at) = half4{(_Float16)o[0], (_Float16)o[1], (_Float16)o[2], (_Float16)o[3]};
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
  // Cut into equal pieces, a tile has less than twice as many as its steps are spans, which are kPieces at most; of a stretch two are kept
  auto of = [&](auto form) {
    using F = decltype(form);
    return pool_of(c).capacity <= F::kUncut * F::kStep ? (int64_t)0 : F::parts(c->n_kv_heads) * F::kPartFloats * 4;
  };
  return kPlanBytes + kCutBytes + (c->head_dim == 128 ? std::max(of(Form<128, true>{}), of(Form<128, false>{})) : std::max(of(Form<64, true>{}), of(Form<64, false>{})));
}

int okv_chunk_attn(const okv_layer_pool *c, const okv_rows *r, const okv_chunk *a, const void *q, int64_t q_stride, void *out, void *stream) {
  const char *const who = "okv_chunk_attn";
  if (const char *why = problem(c, r)) return report(OKV_EINVAL, "%s: %s", who, why);
  if (!a) return report(OKV_EINVAL, "%s: NULL pointer", who);
  // (below 1e-30 a product with them would leave the range of fp32; a quotient above 1e30, whose scores are the cap anyway, is that)
  for (const float x : {a->scale, a->cap})
    if (x != 0.f && !(x >= 1e-30f && x <= 1e30f)) return report(OKV_EINVAL, "%s: scale and cap must be 0 or in [1e-30, 1e30]", who);
  if (a->window < 0) return report(OKV_EINVAL, "%s: window must not be negative", who);
  if (a->out_dtype != 0 && a->out_dtype != 1) return report(OKV_EINVAL, "%s: out_dtype must be 0 or 1", who);
  const int32_t d = c->head_dim;
  if (q_stride < (int64_t)c->n_q_heads * d || q_stride % 8) return report(OKV_EINVAL, "%s: q_stride must be a multiple of 8 and at least n_q_heads * head_dim", who);
  if (r->batch == 0 || r->n_rows == 0) return OKV_OK;
  if (!q || !out) return report(OKV_EINVAL, "%s: NULL pointer", who);
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(a->slopes, 4) || !aligned(a->prefix, 4)) return report(OKV_EINVAL, "%s: q and out must be 16-byte aligned, slopes and prefix 4", who);
  const int64_t need = okv_chunk_workspace_bytes(c);
  if ((!a->workspace || a->workspace_bytes < need || !aligned(a->workspace, 256)))
    return report(OKV_ENOSPC, "%s: the workspace must be %lld bytes, 256-byte aligned", who, (long long)need);
  const Pool pool = pool_of(c);
  const Rows rows{r->seqs, r->starts, r->lens, r->batch, r->n_rows};
  Attend x;
  x.q = static_cast<const _Float16 *>(q), x.out = out, x.q_stride = q_stride;
  const float scale = a->scale != 0.f ? a->scale : 1.f / sqrtf((float)d);
  x.scale = a->cap != 0.f ? 2.f * kLog2e * std::min(scale / a->cap, 1e30f) : scale * kLog2e, x.cap = a->cap * kLog2e;
  x.window = a->window, x.slopes = a->slopes, x.prefix = a->prefix;
  x.plan = static_cast<Plan *>(a->workspace), x.cuts = static_cast<char *>(a->workspace) + kPlanBytes, x.parts = reinterpret_cast<float *>(x.cuts + kCutBytes);
  const bool wide = a->out_dtype == 1, shaped = a->cap != 0.f || a->slopes;
  // How many rows a sequence brings is on the device: by the mean.  Where contexts are short, so many that the wavefronts of a workgroup would walk them one after the other take less time side by side: us of 8
  // sequences of 90 rows, 16 heads x 64, up to 500 keys 15.3 (shared blocks: 21.6), of 128 rows, 8 heads x 128, up to 200 keys 11.3 (15.6), but up to 2000 keys 47 (41)
  const int64_t all_rows = (int64_t)r->n_rows * pool.R;
  const bool few = all_rows <= (pool.capacity <= 1024 ? 128 : 32) * (int64_t)r->batch;
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto run = [&](auto d_, auto few_, auto wide_) {
    constexpr int D = decltype(d_)::value;
    constexpr bool FEW = decltype(few_)::value, WIDE = decltype(wide_)::value;
    using F = Form<D, FEW>;
    x.may_cut = pool.capacity > F::kUncut * F::kStep;
    // a tile of rows begins at a sequence's first row; cutting into equal pieces adds at most kPieces, stretches are kSlots
    const int64_t tiles = (all_rows + F::kRows - 1) / F::kRows + std::min(r->batch, r->n_rows), items = tiles * pool.G;
    const int64_t pieces = !x.may_cut ? items : FEW ? std::max<int64_t>(items, F::stretches(pool.G) * pool.G) : items + F::kPieces;
    if (pieces > 0x7fffffff / 256) return report(OKV_EINVAL, "%s: too many rows for a call", who);
    if (x.may_cut) x.may_cut = (int32_t)items;
    if (r->batch > 64) hipLaunchKernelGGL((plan_kernel<F, FEW>), dim3(1), dim3(kPlanThreads), 0, s, pool, rows, x);
    if (shaped) hipLaunchKernelGGL((chunk_kernel<D, FEW, WIDE, true>), dim3((unsigned)pieces), dim3(F::kThreads), 0, s, pool, rows, x);
    else hipLaunchKernelGGL((chunk_kernel<D, FEW, WIDE, false>), dim3((unsigned)pieces), dim3(F::kThreads), 0, s, pool, rows, x);
    // (tiles that are cut into equal pieces have more steps than a span)
    static_assert(F::kSlots <= kMostCuts && F::kPieces <= kMostCuts, "");
    const int64_t joined = FEW ? F::stretches(pool.G) * pool.G : std::min<int64_t>(F::kPieces, items);
    if (x.may_cut) hipLaunchKernelGGL((join_kernel<D, FEW, WIDE>), dim3((unsigned)(joined * (F::kRows / kJoinRows<D>))), dim3(kJoinThreads), 0, s, pool, x);
    return hip_result(who);
  };
  auto typed = [&](auto d_) {
    if (few) return wide ? run(d_, std::true_type{}, std::true_type{}) : run(d_, std::true_type{}, std::false_type{});
    return wide ? run(d_, std::false_type{}, std::true_type{}) : run(d_, std::false_type{}, std::false_type{});
  };
  return d == 128 ? typed(std::integral_constant<int, 128>{}) : typed(std::integral_constant<int, 64>{});
}

}  // extern "C"
