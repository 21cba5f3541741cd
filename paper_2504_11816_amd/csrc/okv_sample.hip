// From logits to tokens (include/okv_sample.h): probabilities, and drafted tokens held against them, for gfx950.
//
// Probabilities are bound by HBM, 2 or 4 bytes read and 4 written a logit: 320 rows of 131072 fp16 logits 17 us for the pieces' sums (84 MB, 4.9 TB/s) and 38 for the quotients (168 MB written, the
// logits from the memory-side cache).  5 rows of 32000: one launch of 5.9 us.
// Verification reads one row of the target and one of the draft a sequence: 64 sequences of 131072 tokens 14 us (67 MB, 4.8 TB/s), and 7 to find the tokens; 4 of 32000 in one launch of 12.5 us, which is a
// chain of dependent loads (starts, drafts, their probabilities, the row, the part again).  Sums are in 64 bits: an error of 2^-24 of the sum would
// put one draw of 64 from 131072 equal tokens on the wrong side of a border between two.
#include "okv_sample.h"
#include "okv_lanes.h"
#include "okv_report.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "okv.h"

namespace okv {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// Rows begin anywhere: vectors of elements that are aligned as one of them is
typedef float floatx4 __attribute__((ext_vector_type(4), aligned(4)));

// ---- probabilities --------------------------------------------------------------------------------
//
// Every logit is read and every probability written once where a row fits the registers of a workgroup: one launch.  Longer rows are cut into pieces of as many workgroups, in two launches: the
// largest number and the sum of every piece, then the quotients, whose logits come from the memory-side cache.  A wavefront's store is 1 KiB in a row (four numbers a lane; the first launch, which stores
// nothing, reads eight); past the caches they leave the logits there: us of 320 / 64 rows of 131072 fp16 logits 56 / 14.3, stores kept in the caches 69 / 15.6, eight numbers a lane 70 / 17.4
// and past the caches 84 / 19.9, the first launch four a lane 58.6 / 15.3, a workgroup a row in one launch 88 / 29.5.

constexpr int kRowThreads = 1024, kPieceThreads = 256;
constexpr int kEach = 32;                // logits of a thread, in runs
constexpr int kOneLaunch = kRowThreads * kEach;
constexpr int kPieceLogits = kPieceThreads * kEach;

// The largest number of a piece, where it was first, and the sum of 2^((x - largest) by) over it
struct Seen {
  float top, sum;
  int at, unused;
};

template <int RUN, class T>
__device__ __forceinline__ void load_run(const T *x, const int n, float (&to)[RUN]) {      // n of them are there, -infinity for the others
  typedef T numbers __attribute__((ext_vector_type(16 / sizeof(T) < RUN ? 16 / sizeof(T) : RUN), aligned(sizeof(T))));
  constexpr int kVector = sizeof(numbers) / sizeof(T);
  if (n >= RUN) {
#pragma unroll
    for (int k = 0; k < RUN; k += kVector) {
      const numbers v = *reinterpret_cast<const numbers *>(x + k);
#pragma unroll
      for (int i = 0; i < kVector; ++i) to[k + i] = (float)v[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < RUN; ++i) to[i] = i < n ? (float)x[i] : -INFINITY;
}
// ONCE: past the caches, which have the logits of other pieces
template <bool ONCE>
__device__ __forceinline__ void store_run(float *y, const int n, const float (&x)[4]) {
  if (n >= 4) {
    const floatx4 v = {x[0], x[1], x[2], x[3]};
    if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<floatx4 *>(y));
    else *reinterpret_cast<floatx4 *>(y) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) y[i] = x[i];
}

// THREADS threads' numbers of a piece of a row, RUN from RUN (i THREADS + thread) on each: their largest, first place (at temperature 0), exponentials in their stead, and the sum
template <int THREADS, int RUN>
__device__ __forceinline__ Seen seen_by_all(float (&x)[kEach / RUN][RUN], const float t, const float by, float *shared) {
  constexpr int kWaves = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Seen s{-INFINITY, 0.f, 0x7fffffff, 0};
#pragma unroll
  for (int i = 0; i < kEach / RUN; ++i)
#pragma unroll
    for (int j = 0; j < RUN; ++j) s.top = fmaxf(s.top, x[i][j]);
  s.top = wave_max(s.top);
  if (lane == 0) shared[wave] = s.top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s.top = fmaxf(s.top, shared[w]);
  __syncthreads();
  if (t == 0.f) {
#pragma unroll
    for (int i = kEach / RUN - 1; i >= 0; --i)
#pragma unroll
      for (int j = RUN - 1; j >= 0; --j)
        if (x[i][j] == s.top) s.at = RUN * (i * THREADS + (int)threadIdx.x) + j;
#pragma unroll
    for (int o = 32; o; o >>= 1) s.at = min(s.at, __shfl_xor(s.at, o));
    if (lane == 0) shared[wave] = __builtin_bit_cast(float, s.at);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s.at = min(s.at, __builtin_bit_cast(int, shared[w]));
    if (s.top == -INFINITY) s.at = 0x7fffffff;           // (nothing is the largest)
    return s;
  }
  const float less = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
  for (int i = 0; i < kEach / RUN; ++i)
#pragma unroll
    for (int j = 0; j < RUN; ++j) s.sum += x[i][j] = __builtin_amdgcn_exp2f((x[i][j] - less) * by);
  s.sum = wave_sum(s.sum);
  if (lane == 0) shared[wave] = s.sum;
  __syncthreads();
  s.sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s.sum += shared[w];
  return s;
}
// (x - top) / t in units of log 2.  A temperature below 1e-30 is as good as that: the largest take all.  Of an infinite one the smallest number there is stays, with which differences of finite logits come
// to less than 2^-20 and those of -infinity (0 times which is NaN) to that.
__device__ __forceinline__ float per_temperature(const float t) { return t >= 0.f ? fmaxf(kLog2e / fmaxf(t, 1e-30f), 0x1p-149f) : NAN; }

template <class T>
__global__ void __launch_bounds__(kRowThreads) row_probs_kernel(const T *logits, const int64_t stride, const float *temperature, float *out, const int64_t out_stride, const int vocab) {
  __shared__ float shared[kRowThreads / 64];
  const T *x = logits + blockIdx.x * stride;
  float *y = out + blockIdx.x * out_stride;
  float v[kEach / 4][4];
#pragma unroll
  for (int i = 0; i < kEach / 4; ++i) {
    const int at = 4 * (i * kRowThreads + (int)threadIdx.x);
    load_run(x + at, vocab - at, v[i]);
  }
  const float t = temperature ? temperature[blockIdx.x] : 1.f;
  const Seen s = seen_by_all<kRowThreads, 4>(v, t, per_temperature(t), shared);
  const float over = s.sum == 0.f ? 0.f : 1.f / s.sum;
#pragma unroll
  for (int i = 0; i < kEach / 4; ++i) {
    const int at = 4 * (i * kRowThreads + (int)threadIdx.x);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = t == 0.f ? (at + j == s.at ? 1.f : 0.f) : v[i][j] * over;
    store_run<false>(y + at, vocab - at, v[i]);
  }
}

template <class T>
__global__ void __launch_bounds__(kPieceThreads) piece_seen_kernel(const T *logits, const int64_t stride, const float *temperature, const int vocab, Seen *seen) {
  __shared__ float shared[kPieceThreads / 64];
  const int first = blockIdx.x * kPieceLogits, row = blockIdx.y;
  const T *x = logits + row * stride;
  float v[kEach / 8][8];
#pragma unroll
  for (int i = 0; i < kEach / 8; ++i) {
    const int at = first + 8 * (i * kPieceThreads + (int)threadIdx.x);
    load_run(x + at, vocab - at, v[i]);
  }
  const float t = temperature ? temperature[row] : 1.f;
  Seen s = seen_by_all<kPieceThreads, 8>(v, t, per_temperature(t), shared);
  if (s.at != 0x7fffffff) s.at += first;
  if (threadIdx.x == 0) seen[(int64_t)row * gridDim.x + blockIdx.x] = s;
}
template <bool ONCE, class T>
__global__ void __launch_bounds__(kPieceThreads) piece_probs_kernel(const T *logits, const int64_t stride, const float *temperature, float *out, const int64_t out_stride, const int vocab,
                                                                    const Seen *seen) {
  const int first = blockIdx.x * kPieceLogits, row = blockIdx.y, lane = threadIdx.x & 63, pieces = gridDim.x;
  const T *x = logits + row * stride;
  float *y = out + row * out_stride;
  float v[kEach / 4][4];
#pragma unroll
  for (int i = 0; i < kEach / 4; ++i) {
    const int at = first + 4 * (i * kPieceThreads + (int)threadIdx.x);
    load_run(x + at, vocab - at, v[i]);
  }
  const float t = temperature ? temperature[row] : 1.f, by = per_temperature(t);
  float top = -INFINITY, sum = 0.f;
  int at_top = 0x7fffffff;
  for (int i = lane; i < pieces; i += 64) top = fmaxf(top, seen[(int64_t)row * pieces + i].top);
  top = wave_max(top);
  const float less = top == -INFINITY ? 0.f : top;
  for (int i = lane; i < pieces; i += 64) {
    const Seen s = seen[(int64_t)row * pieces + i];
    if (s.top == top) at_top = min(at_top, s.at);
    sum += s.top == -INFINITY ? s.sum : s.sum * __builtin_amdgcn_exp2f((s.top - less) * by);
  }
  sum = wave_sum(sum);
#pragma unroll
  for (int o = 32; o; o >>= 1) at_top = min(at_top, __shfl_xor(at_top, o));
  const float over = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int i = 0; i < kEach / 4; ++i) {
    const int at = first + 4 * (i * kPieceThreads + (int)threadIdx.x);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] = t == 0.f ? (at + j == at_top ? 1.f : 0.f) : __builtin_amdgcn_exp2f((v[i][j] - less) * by) * over;
    store_run<ONCE>(y + at, vocab - at, v[i]);
  }
}

// ---- verification ---------------------------------------------------------------------------------

struct Verify {
  const float *target, *draft;
  int64_t target_stride, draft_stride;
  const int32_t *drafts, *starts;
  const float *uniforms;
  int32_t *tokens, *accepted, *rejected;
  int32_t batch, n_rows, vocab;
};

// A sequence's rows, and how many of its drafts are accepted: by a wavefront
struct Turn {
  int first, n, accepted;
};
__device__ __forceinline__ Turn rows_of(const Verify &a, const int b) {
  Turn t;
  t.first = min(max(a.starts[b], 0), a.n_rows);
  t.n = min(max(a.starts[b + 1], t.first), a.n_rows) - t.first;
  t.accepted = t.n;
  return t;
}
__device__ __forceinline__ Turn turn_of(const Verify &a, const int b) {
  const int lane = threadIdx.x & 63;
  Turn t = rows_of(a, b);
  for (int i0 = 0; i0 < t.n; i0 += 64) {
    const int i = i0 + lane;
    bool bad = false;
    if (i < t.n) {
      const int64_t at = t.first + i;
      const int x = a.drafts[at];
      bad = true;
      if (x >= 0 && x < a.vocab) {
        const float q = a.draft ? a.draft[at * a.draft_stride + x] : 1.f;
        bad = !(__fmul_rn(a.uniforms[at + b], q) < a.target[(at + b) * a.target_stride + x]);
      }
    }
    const uint64_t stop = __ballot(bad);
    if (stop) {
      t.accepted = i0 + __ffsll((unsigned long long)stop) - 1;
      break;
    }
  }
  return t;
}

// Weights of the row that the next token is drawn from, kPart tokens at a time, 32 in each lane of a wavefront: four at a time side by side (to be added up), or one after the other (to find a
// token; 64 lanes' 32 in a row are 64 lines a load)
constexpr int kPart = 2048, kOfLane = kPart / 64;
template <bool IN_A_ROW>
struct Weights {
  float p[kOfLane], q[kOfLane];
  int without, i0;                       // the token that a certain draft takes off, -1: none; this lane's first
  __device__ __forceinline__ static int place(const int i) { return IN_A_ROW ? i : i / 4 * 256 + i % 4; }      // of a lane's i-th behind its first
  __device__ __forceinline__ Weights(const Verify &a, const int b, const Turn &t, const int part) {
    const int64_t at = t.first + t.accepted;
    i0 = part * kPart + (int)(threadIdx.x & 63) * (IN_A_ROW ? kOfLane : 4);
    const bool rejected = t.accepted < t.n;
    read(p, a.target + (at + b) * a.target_stride + i0, a.vocab - i0);
    if (rejected && a.draft) read(q, a.draft + at * a.draft_stride + i0, a.vocab - i0);
    else
#pragma unroll
      for (int i = 0; i < kOfLane; ++i) q[i] = 0.f;
    without = rejected && !a.draft ? a.drafts[at] : -1;
  }
  __device__ __forceinline__ static void read(float (&to)[kOfLane], const float *from, const int n) {
#pragma unroll
    for (int i = 0; i < kOfLane; i += 4) {
      if (place(i) + 4 <= n) {
        const floatx4 v = *reinterpret_cast<const floatx4 *>(from + place(i));
#pragma unroll
        for (int j = 0; j < 4; ++j) to[i + j] = v[j];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[i + j] = place(i) + j < n ? from[place(i) + j] : 0.f;
      }
    }
  }
  __device__ __forceinline__ static double counted(const double w) { return w > 0. && w < INFINITY ? w : 0.; }
  __device__ __forceinline__ double one(const int i, const bool all) const { return counted(all ? p[i] : i0 + place(i) == without ? 0. : (double)p[i] - (double)q[i]); }
};
// A part's sum: of what the target has above the draft, or (all) of the target
__device__ __forceinline__ double sum_of(const Verify &a, const int b, const Turn &t, const int part, const bool all) {
  const Weights<false> w(a, b, t, part);
  double sum = 0.;
#pragma unroll
  for (int i = 0; i < kOfLane; ++i) sum += w.one(i, all);
  return wave_sum(sum);
}
// The first lane whose `mine` and those before it come to more than x less `before`, and the sum before it; should rounding leave none, the last that is not 0 (-1: all are)
__device__ __forceinline__ int lane_of(const double mine, const double x, double &before) {
  const double upto = wave_scan(mine);
  const uint64_t above = __ballot(mine > 0. && before + upto > x), some = __ballot(mine > 0.);
  const int at = above ? __ffsll((unsigned long long)above) - 1 : 63 - __clzll((long long)some);
  before += above ? lane_value(upto - mine, at) : lane_value(upto, 63);
  return above ? at : some ? at | 64 : -1;             // (| 64: of those so far)
}
// Where u lies among the parts' sums, by a wavefront: the part (-1: all sums are 0), the sum before it (below 0: rounding has left none, it is the last part with a weight and its last token),
// and u times the sum of them
struct Place {
  int part;
  double before, x;
};
__device__ __forceinline__ Place place_of(const double *sums, const int parts, const float u) {
  const int lane = threadIdx.x & 63;
  double total = 0.;
  for (int i = lane; i < parts; i += 64) total += sums[i];
  Place p{-1, 0., (double)u * wave_sum(total)};
  for (int i0 = 0; i0 < parts; i0 += 64) {
    const int at = lane_of(i0 + lane < parts ? sums[i0 + lane] : 0., p.x, p.before);
    if (at < 0) continue;
    p.part = i0 + (at & 63);
    if (at < 64) return p;
  }
  p.before = -1.;
  return p;
}
// The token in its part, by a wavefront that has the part's weights
__device__ __forceinline__ int token_in(const Weights<true> &w, const Place &p, const bool all) {
  double mine = 0.;
#pragma unroll
  for (int i = 0; i < kOfLane; ++i) mine += w.one(i, all);
  const bool last = p.before < 0.;
  double before = last ? 0. : p.before;
  const double x = last ? INFINITY : p.x;
  const int at = lane_of(mine, x, before);
  // (lane `at` goes through its weights)
  int token = 0;
  bool found = false;
#pragma unroll
  for (int i = 0; i < kOfLane; ++i) {
    const double v = w.one(i, all);
    before += v;
    if (v > 0. && !found) token = i, found = at < 64 && before > x;
  }
  return p.part * kPart + (at & 63) * kOfLane + lane_value(token, at & 63);
}
// The token that u draws, by a wavefront, from the parts' sums
__device__ __forceinline__ int next_token(const Verify &a, const int b, const Turn &t, const double *sums, const int parts, const float u) {
  Place p = place_of(sums, parts, u);
  const bool fallback = p.part < 0;
  if (fallback) {                                        // nothing above the draft: from all of the target
    double x = 0.;
    for (int part = 0; part < parts; ++part) x += sum_of(a, b, t, part, true);
    p.x = (double)u * x, p.before = 0.;
    int last = -1;
    for (int part = 0; part < parts; ++part) {
      const double sum = sum_of(a, b, t, part, true);
      if (sum > 0.) last = part;
      if (sum > 0. && p.before + sum > p.x) {
        p.part = part;
        break;
      }
      p.before += sum;
    }
    if (p.part < 0) p.part = last, p.before = -1.;
  }
  if (p.part < 0) return -1;
  const Weights<true> w(a, b, t, p.part);
  return token_in(w, p, fallback);
}
__device__ __forceinline__ void write_tokens(const Verify &a, const int b, const Turn &t, const int token) {
  const int lane = threadIdx.x & 63;
  for (int i = lane; i <= t.n; i += 64) a.tokens[t.first + b + i] = i < t.accepted ? a.drafts[t.first + i] : i == t.accepted ? token : -1;
  if (lane == 0) {
    a.accepted[b] = t.accepted;
    if (a.rejected) a.rejected[b] = t.n - t.accepted;
  }
}

// A workgroup per sequence, in one launch: few tokens
constexpr int kOneWaves = 8, kOneParts = 16;
__global__ void __launch_bounds__(64 * kOneWaves) verify_kernel(Verify a) {
  __shared__ double sums[kOneParts];
  const int b = blockIdx.x, wave = threadIdx.x >> 6, parts = (a.vocab + kPart - 1) / kPart;
  const Turn t = turn_of(a, b);
  const float u = a.uniforms[t.first + b + t.n];
  for (int part = wave; part < parts; part += kOneWaves) {
    const double sum = sum_of(a, b, t, part, false);
    if ((threadIdx.x & 63) == 0) sums[part] = sum;
  }
  __syncthreads();
  if (wave == 0) write_tokens(a, b, t, next_token(a, b, t, sums, parts, u));
}

// Many tokens: a wavefront per part of every sequence, then one per sequence.  sums [batch][parts]
constexpr int kPartWaves = 4;
__global__ void __launch_bounds__(64 * kPartWaves) parts_kernel(Verify a, double *sums) {
  const int b = blockIdx.y, part = blockIdx.x * kPartWaves + (threadIdx.x >> 6), parts = (a.vocab + kPart - 1) / kPart;
  if (part >= parts) return;
  const Turn t = turn_of(a, b);
  const double sum = sum_of(a, b, t, part, false);
  if ((threadIdx.x & 63) == 0) {
    sums[(int64_t)b * parts + part] = sum;
    if (part == 0) a.accepted[b] = t.accepted;
  }
}
__global__ void __launch_bounds__(64) token_kernel(Verify a, const double *sums) {
  const int b = blockIdx.x, parts = (a.vocab + kPart - 1) / kPart;
  Turn t = rows_of(a, b);
  t.accepted = min(max(a.accepted[b], 0), t.n);
  const float u = a.uniforms[t.first + b + t.n];
  write_tokens(a, b, t, next_token(a, b, t, sums + (int64_t)b * parts, parts, u));
}

bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
int hip_result(const char *who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OKV_OK : report(OKV_EHIP, "%s: %s", who, hipGetErrorString(e));
}

}  // namespace

}  // namespace okv

using namespace okv;

extern "C" {

int64_t okv_token_probs_workspace_bytes(int32_t max_rows, int32_t vocab) {
  if (max_rows < 0 || max_rows > OKV_SAMPLE_MAX_ROWS || vocab < 1 || vocab > OKV_SAMPLE_MAX_VOCAB)
    return report(OKV_EINVAL, "okv_token_probs_workspace_bytes: rows must be in [0, 2^20] and vocab in [1, 2^24]");
  return vocab <= kOneLaunch ? 0 : (int64_t)max_rows * ((vocab + kPieceLogits - 1) / kPieceLogits) * (int64_t)sizeof(Seen);
}

int okv_token_probs(const void *logits, int32_t dtype, int64_t stride, const float *temperature, float *out, int64_t out_stride, int32_t rows, int32_t vocab,
                    void *workspace, int64_t workspace_bytes, void *stream) {
  const char *const who = "okv_token_probs";
  const int64_t need = okv_token_probs_workspace_bytes(rows, vocab);
  if (need < 0) return (int)need;
  if (dtype != 0 && dtype != 1) return report(OKV_EINVAL, "%s: dtype must be 0 or 1", who);
  if (stride < vocab || out_stride < vocab) return report(OKV_EINVAL, "%s: rows must be at least vocab elements apart", who);
  if (rows == 0) return OKV_OK;
  if (!logits || !out || !aligned(logits, dtype ? 4 : 2) || !aligned(out, 4) || !aligned(temperature, 4)) return report(OKV_EINVAL, "%s: NULL or misaligned pointer", who);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return report(OKV_ENOSPC, "%s: the workspace must be %lld bytes, 16-byte aligned", who, (long long)need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto run = [&](auto *x) {
    if (vocab <= kOneLaunch) {
      hipLaunchKernelGGL(row_probs_kernel, dim3((unsigned)rows), dim3(kRowThreads), 0, s, x, stride, temperature, out, out_stride, vocab);
      return;
    }
    Seen *const seen = static_cast<Seen *>(workspace);
    const int32_t pieces = (vocab + kPieceLogits - 1) / kPieceLogits;
    for (int32_t first = 0; first < rows; first += 32768) {      // (rows of a grid's second dimension)
      const dim3 grid((unsigned)pieces, (unsigned)std::min(rows - first, 32768));
      const float *const t = temperature ? temperature + first : nullptr;
      Seen *const at = seen + (int64_t)first * pieces;
      hipLaunchKernelGGL(piece_seen_kernel, grid, dim3(kPieceThreads), 0, s, x + first * stride, stride, t, vocab, at);
      // (of 256 rows of 50001, most of which are not aligned: 22 us, past the caches 24)
      auto probs = [&](auto once) {
        hipLaunchKernelGGL((piece_probs_kernel<decltype(once)::value>), grid, dim3(kPieceThreads), 0, s, x + first * stride, stride, t, out + first * out_stride, out_stride, vocab, static_cast<const Seen *>(at));
      };
      if (aligned(out, 16) && out_stride % 4 == 0) probs(std::true_type{});
      else probs(std::false_type{});
    }
  };
  if (dtype == 0) run(static_cast<const _Float16 *>(logits));
  else run(static_cast<const float *>(logits));
  return hip_result(who);
}

int64_t okv_verify_workspace_bytes(int32_t max_batch, int32_t vocab) {
  if (max_batch < 0 || max_batch > OKV_VERIFY_MAX_BATCH || vocab < 1 || vocab > OKV_SAMPLE_MAX_VOCAB)
    return report(OKV_EINVAL, "okv_verify_workspace_bytes: batch must be in [0, 4096] and vocab in [1, 2^24]");
  return (int64_t)max_batch * ((vocab + kPart - 1) / kPart) * 8;
}

int okv_verify(const float *target, int64_t target_stride, const float *draft_probs, int64_t draft_stride, const int32_t *drafts, const int32_t *starts,
               const float *uniforms, int32_t *tokens, int32_t *accepted, int32_t *rejected, int32_t batch, int32_t n_rows, int32_t vocab, void *workspace,
               int64_t workspace_bytes, void *stream) {
  const char *const who = "okv_verify";
  const int64_t need = okv_verify_workspace_bytes(batch, vocab);
  if (need < 0) return (int)need;
  if (n_rows < 0) return report(OKV_EINVAL, "%s: n_rows must not be negative", who);
  if (target_stride < vocab || (draft_probs && draft_stride < vocab)) return report(OKV_EINVAL, "%s: rows must be at least vocab elements apart", who);
  if (batch == 0) return OKV_OK;
  if (!target || !starts || !uniforms || !tokens || !accepted || (n_rows && !drafts)) return report(OKV_EINVAL, "%s: NULL pointer", who);
  for (const void *p : {static_cast<const void *>(target), static_cast<const void *>(draft_probs), static_cast<const void *>(drafts), static_cast<const void *>(starts),
                        static_cast<const void *>(uniforms), static_cast<const void *>(tokens), static_cast<const void *>(accepted), static_cast<const void *>(rejected)})
    if (!aligned(p, 4)) return report(OKV_EINVAL, "%s: misaligned pointer", who);
  if (!workspace || workspace_bytes < need || !aligned(workspace, 16)) return report(OKV_ENOSPC, "%s: the workspace must be %lld bytes, 16-byte aligned", who, (long long)need);
  Verify a{target, draft_probs, target_stride, draft_stride, drafts, starts, uniforms, tokens, accepted, rejected, batch, n_rows, vocab};
  const int32_t parts = (vocab + kPart - 1) / kPart;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (parts <= kOneParts) {
    hipLaunchKernelGGL(verify_kernel, dim3((unsigned)batch), dim3(64 * kOneWaves), 0, s, a);
  } else {
    hipLaunchKernelGGL(parts_kernel, dim3((unsigned)((parts + kPartWaves - 1) / kPartWaves), (unsigned)batch), dim3(64 * kPartWaves), 0, s, a, static_cast<double *>(workspace));
    hipLaunchKernelGGL(token_kernel, dim3((unsigned)batch), dim3(64), 0, s, a, static_cast<const double *>(workspace));
  }
  return hip_result(who);
}

}  // extern "C"
