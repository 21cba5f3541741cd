// From logits to tokens (include/okv_sample.h): probabilities, and drafted tokens held against them, for gfx950.
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
constexpr int kThreads = 1024, kWaves = kThreads / 64;

// ---- probabilities --------------------------------------------------------------------------------

// The largest number of a row so far, the sum of 2^((x - largest) by) over it, and where it was first
struct Seen {
  float top, sum;
  int at;
};
__device__ __forceinline__ Seen joined(const Seen &a, const Seen &b, const float by) {
  Seen r;
  r.top = fmaxf(a.top, b.top);
  // (-infinity alone has nothing to add)
  r.sum = (a.top == -INFINITY ? a.sum : a.sum * __builtin_amdgcn_exp2f((a.top - r.top) * by)) + (b.top == -INFINITY ? b.sum : b.sum * __builtin_amdgcn_exp2f((b.top - r.top) * by));
  r.at = a.top > b.top || (a.top == b.top && a.at < b.at) ? a.at : b.at;
  return r;
}
__device__ __forceinline__ Seen of_workgroup(Seen x, const float by, Seen *waves) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = joined(x, Seen{__shfl_xor(x.top, o), __shfl_xor(x.sum, o), __shfl_xor(x.at, o)}, by);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  x = waves[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) x = joined(x, waves[w], by);
  return x;
}

template <class T>
__global__ void __launch_bounds__(kThreads) probs_kernel(const T *logits, const int64_t stride, const float *temperature, float *out, const int64_t out_stride,
                                                         const int vocab) {
  __shared__ Seen waves[kWaves];
  const T *x = logits + blockIdx.x * stride;
  float *y = out + blockIdx.x * out_stride;
  const float t = temperature ? temperature[blockIdx.x] : 1.f;
  // (x - top) / t in units of log 2.  A temperature below 1e-30 is as good as none: the largest take all
  const float by = t >= 0.f ? kLog2e / fmaxf(t, 1e-30f) : NAN;
  Seen s{-INFINITY, 0.f, 0x7fffffff};
  for (int i = threadIdx.x; i < vocab; i += kThreads) {
    const float v = (float)x[i];
    if (v > s.top) s = Seen{v, s.top == -INFINITY ? s.sum + 1.f : s.sum * __builtin_amdgcn_exp2f((s.top - v) * by) + 1.f, i};
    else if (v != -INFINITY) s.sum += __builtin_amdgcn_exp2f((v - s.top) * by);
  }
  s = of_workgroup(s, by, waves);
  if (t == 0.f) {
    for (int i = threadIdx.x; i < vocab; i += kThreads) y[i] = i == s.at ? 1.f : 0.f;
    return;
  }
  const float over = s.sum == 0.f ? 0.f : 1.f / s.sum;
  for (int i = threadIdx.x; i < vocab; i += kThreads) {
    const float v = (float)x[i];
    y[i] = v == -INFINITY && s.sum == s.sum ? 0.f : __builtin_amdgcn_exp2f((v - s.top) * by) * over;
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

__device__ __forceinline__ bool counts(const double w) { return w > 0. && w < INFINITY; }

// A sequence's rows, how many of its drafts are accepted, and where its next token is drawn from: what a wavefront finds out
struct Turn {
  int first, n, accepted;
};
__device__ __forceinline__ Turn turn_of(const Verify &a, const int b) {
  const int lane = threadIdx.x & 63;
  Turn t;
  t.first = min(max(a.starts[b], 0), a.n_rows);
  t.n = min(max(a.starts[b + 1], t.first), a.n_rows) - t.first;
  t.accepted = t.n;
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

// The weights of the row that the next token is drawn from
struct Weights {
  const float *p, *q;                    // q NULL: nothing is taken off, but the whole of `without`
  int without;
  __device__ __forceinline__ Weights(const Verify &a, const int b, const Turn &t) {
    const int64_t at = t.first + t.accepted;
    p = a.target + (at + b) * a.target_stride;
    q = t.accepted < t.n && a.draft ? a.draft + at * a.draft_stride : nullptr;
    without = t.accepted < t.n && !a.draft ? a.drafts[at] : -1;
  }
  __device__ __forceinline__ double rest(const int i) const {
    const double w = i == without ? 0. : q ? (double)p[i] - (double)q[i] : (double)p[i];
    return counts(w) ? w : 0.;
  }
  __device__ __forceinline__ double all(const int i) const { return counts(p[i]) ? (double)p[i] : 0.; }
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Tokens kPart at a time: sums over these in 64 bits, then the part in which u times the sum lies, then the token
constexpr int kPart = 2048;

__device__ __forceinline__ void write_tokens(const Verify &a, const int b, const Turn &t, const int token) {
  const int lane = threadIdx.x & 63;
  for (int i = lane; i <= t.n; i += 64) a.tokens[t.first + b + i] = i < t.accepted ? a.drafts[t.first + i] : i == t.accepted ? token : -1;
  if (lane == 0) {
    a.accepted[b] = t.accepted;
    if (a.rejected) a.rejected[b] = t.n - t.accepted;
  }
}

// The token, by one wavefront: sums[part] are over rest(), sums[parts + part] over all()
__device__ __forceinline__ int token_of(const Verify &a, const Weights &w, const double *sums, const int parts, const float u) {
  const int lane = threadIdx.x & 63;
  double total = 0.;
  for (int i = lane; i < parts; i += 64) total += sums[i];
  total = wave_sum64(total);
  const bool fallback = !(total > 0.);
  if (fallback) {
    total = 0.;
    sums += parts;
    for (int i = lane; i < parts; i += 64) total += sums[i];
    total = wave_sum64(total);
    if (!(total > 0.)) return -1;
  }
  const double x = (double)u * total;
  // the first place whose sum up to it is above x; should rounding leave none, the last whose weight is not 0
  auto find = [&](const int n, const auto &weight, double &before) {
    int last = -1;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const double v = i0 + lane < n ? weight(i0 + lane) : 0.;
      double upto = v;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double other = __shfl_up(upto, o);
        if (lane >= o) upto += other;
      }
      const uint64_t there = __ballot(v > 0.), above = __ballot(v > 0. && before + upto > x);
      if (above) {
        const int at = __ffsll((unsigned long long)above) - 1;
        before += __shfl(upto - v, at);
        return i0 + at;
      }
      if (there) last = i0 + 63 - __clzll((long long)there);
      before += __shfl(upto, 63);
    }
    return last;
  };
  double before = 0.;
  const int part = find(parts, [&](int i) { return sums[i]; }, before);
  if (part < 0) return -1;
  const int i0 = part * kPart, n = min(kPart, a.vocab - i0);
  if (before > x) before = x;
  return i0 + find(n, [&](int i) { return fallback ? w.all(i0 + i) : w.rest(i0 + i); }, before);
}

// A workgroup per sequence
__global__ void __launch_bounds__(kThreads) verify_kernel(Verify a, double *sums) {
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int parts = (a.vocab + kPart - 1) / kPart;
  double *mine = sums + (int64_t)b * 2 * parts;
  const Turn t = turn_of(a, b);
  const Weights w(a, b, t);
  for (int part = wave; part < parts; part += kWaves) {
    double rest = 0., all = 0.;
#pragma unroll 4
    for (int i = part * kPart + lane; i < min((part + 1) * kPart, a.vocab); i += 64) rest += w.rest(i), all += w.all(i);
    rest = wave_sum64(rest), all = wave_sum64(all);
    if (lane == 0) mine[part] = rest, mine[parts + part] = all;
  }
  __threadfence_block();
  __syncthreads();
  if (wave) return;
  write_tokens(a, b, t, token_of(a, w, mine, parts, a.uniforms[t.first + b + t.n]));
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
  return 0;
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
  const dim3 grid((unsigned)rows), block(kThreads);
  if (dtype == 0)
    hipLaunchKernelGGL(probs_kernel<_Float16>, grid, block, 0, static_cast<hipStream_t>(stream), static_cast<const _Float16 *>(logits), stride, temperature, out, out_stride, vocab);
  else
    hipLaunchKernelGGL(probs_kernel<float>, grid, block, 0, static_cast<hipStream_t>(stream), static_cast<const float *>(logits), stride, temperature, out, out_stride, vocab);
  return hip_result(who);
}

int64_t okv_verify_workspace_bytes(int32_t max_batch, int32_t vocab) {
  if (max_batch < 0 || max_batch > OKV_VERIFY_MAX_BATCH || vocab < 1 || vocab > OKV_SAMPLE_MAX_VOCAB)
    return report(OKV_EINVAL, "okv_verify_workspace_bytes: batch must be in [0, 4096] and vocab in [1, 2^24]");
  return (int64_t)max_batch * 2 * ((vocab + kPart - 1) / kPart) * 8;
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
  hipLaunchKernelGGL(verify_kernel, dim3((unsigned)batch), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, static_cast<double *>(workspace));
  return hip_result(who);
}

}  // extern "C"
