// Linear layers with 4-bit weights (include/okv_linear4.h), for gfx950.
//
// y[m][n] = sum_g scale[n][g] sum_{k in g} x[m][k] (code[n][k] - zero[n][g]) for a decode batch's few rows: bound by reading the codes.
//
//   * one 16-byte load per lane brings a wavefront a block of 16 features x 128 inputs, in operand order for four 16x16x32
//     matrix-core instructions: nothing moves between lanes;
//   * a code becomes an fp16 number with one and-or (0x6400 | code is 1024 + code, a method that is widely published; four bits further up it is 1024 + 16 code) and one packed
//     subtraction or fused multiply-add that also takes the zero point off: code - zero, exactly, at about one instruction a weight;
//   * the sums of a group stay apart from the others' in fp32 and are multiplied by its scale there: one fma per result and group
//     instead of one rounding per weight;
//   * the rows of x are fetched by every wavefront for itself, in operand order, through L2: their bytes are x times the number of tiles a
//     workgroup leaves apart.  So a workgroup takes several tiles of features (1 to 8) and, where that leaves compute units idle, only a cut of
//     the inputs; its wavefronts take blocks of 128 inputs in turn and add up through LDS.  (Rows staged in LDS for the whole workgroup,
//     with a barrier per round of blocks, were 10 to 30 % slower from 16 to 256 rows.)
//
// Measured, codes from HBM, groups of 128, us: 1 row x 16384 x 4096 10.2 (34.6 MB: 3.4 TB/s), 12288 x 4096 8.7, 4096 x 4096 4.9, 4096 x 16384 11.5;
// 32 rows 15.7, 13.9, 10.2, 18.9; 256 rows x 16384 x 4096 62.6 (0.55 PFLOP/s).
#include "okv_linear4.h"
#include "okv_report.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "okv.h"

namespace okv {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlockIn = 128;            // inputs of a block

struct Linear4Args {
  const _Float16 *x;
  const u32x4 *codes;                    // [n_out / 16][blocks][64]
  const _Float16 *scales;                // [n_out / 16][blocks][4][groups of a block][4]
  const uint8_t *zeros;                  // [n_out / 16][blocks][16][groups of a block]
  const _Float16 *bias, *residual;
  _Float16 *out[3];
  int32_t end[3];                        // first feature behind run s
  int32_t m, n_out, n_in, blocks, relu;
  float *shares;                         // [cuts][m][n_out] where the inputs are cut over workgroups
  int32_t cuts;
};

// y + bias, ReLU, residual, rounding, and where it goes: 4 consecutive features n .. of a row
__device__ __forceinline__ void finish(const Linear4Args &a, floatx4 y, const int row, const int n) {
  if (a.bias) {
    const half4v bias = *reinterpret_cast<const half4v *>(a.bias + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += (float)bias[e];
  }
  if (a.relu)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = y[e] < 0.f ? 0.f : y[e];      // (NaN stays)
  if (a.residual) {
    const half4v more = *reinterpret_cast<const half4v *>(a.residual + (int64_t)row * a.n_out + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += (float)more[e];
  }
  const int s = n < a.end[0] ? 0 : n < a.end[1] ? 1 : 2, first = s == 0 ? 0 : s == 1 ? a.end[0] : a.end[1];
  _Float16 *to = s == 0 ? a.out[0] : s == 1 ? a.out[1] : a.out[2];
  const int width = (s == 0 ? a.end[0] : s == 1 ? a.end[1] : a.end[2]) - first;
  half4v h;
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = (_Float16)y[e];
  *reinterpret_cast<half4v *>(to + (int64_t)row * width + n - first) = h;
}

// 8 codes -> code - zero.  near: -(1024 + zero) twice, far: -(64 + zero) twice
__device__ __forceinline__ half8 unpack4bit(const uint32_t w, const half2v near, const half2v far) {
  const half2v by = {(_Float16)0.0625f, (_Float16)0.0625f};
  const uint32_t v = w >> 8;
  const half2v a = __builtin_bit_cast(half2v, (w & 0x000f000fu) | 0x64006400u) + near;
  const half2v b = __builtin_elementwise_fma(__builtin_bit_cast(half2v, (w & 0x00f000f0u) | 0x64006400u), by, far);
  const half2v c = __builtin_bit_cast(half2v, (v & 0x000f000fu) | 0x64006400u) + near;
  const half2v d = __builtin_elementwise_fma(__builtin_bit_cast(half2v, (v & 0x00f000f0u) | 0x64006400u), by, far);
  return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The value N lanes before, around the row of 16 lanes
template <int N>
__device__ __forceinline__ half8 turn(const half8 x) {
  u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[i], 0x120 + N, 0xf, 0xf, false);
  return __builtin_bit_cast(half8, w);
}

template <class T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Few {
  T v[N];
};

// MF fragments of 16 rows and NT tiles of 16 features per workgroup, WAVES wavefronts that take the blocks of 128 inputs in turn, DEPTH blocks in
// flight each; GROUPS groups in a block.  Workgroups (x, y, z): tiles, cuts of the inputs, rows.
// FOUR: up to 4 rows.  What bounds few rows is the number of loads, and a fragment's four loads bring 4 rows' 16 bytes a lane four times over:
// one load brings all of a block's 128 inputs, lane 4 j + i of a row of 16 lanes row i's part of product j, which turns into place by 4 j
// lanes.  us, 1 row, without it and with it: 4096 x 16384 14.3 and 11.8, 4096 x 4096 5.4 and 4.9.
template <int MF, int NT, int WAVES, int DEPTH, bool FOUR, int GROUPS, bool ZEROS>
__global__ void __launch_bounds__(64 * WAVES) linear4_kernel(Linear4Args a) {
  __shared__ floatx4 shares[WAVES][MF * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile0 = blockIdx.x * NT, row0 = blockIdx.z * 16 * MF, n_tiles = a.n_out / 16;
  const int first = (int)((int64_t)a.blocks * blockIdx.y / a.cuts), last = (int)((int64_t)a.blocks * (blockIdx.y + 1) / a.cuts);
  const int r = lane % 16, quarter = lane / 16;
  // Where there are many results, one tile after the other: the compiler would issue all their products first and spill.  (The empty
  // assembly statements keep their order.)
  constexpr bool kApart = GROUPS == 4 ? MF * NT > 2 : GROUPS == 2 && MF * NT >= 12;
  floatx4 sum[MF][NT] = {};
  const _Float16 *row[MF];               // rows that there are not are the last one: what they give is not stored
#pragma unroll
  for (int f = 0; f < MF; ++f) row[f] = a.x + (int64_t)min(row0 + 16 * f + (FOUR ? r % 4 : r), a.m - 1) * a.n_in + (FOUR ? 32 * (r / 4) : 0) + 8 * quarter;
  struct Block {
    u32x4 w[NT];
    Few<u32x2, GROUPS> scale[NT];
    Few<uint8_t, GROUPS> zero[NT];
    half8 x[MF][FOUR ? 1 : 4];
  } in[DEPTH];
  const half8 none = {};
  const auto load = [&](Block &k, const int b) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int64_t at = (int64_t)min(tile0 + t, n_tiles - 1) * a.blocks + b;
      k.w[t] = __builtin_nontemporal_load(a.codes + at * 64 + lane);
      k.scale[t] = *reinterpret_cast<const Few<u32x2, GROUPS> *>(a.scales + (at * 4 + quarter) * 4 * GROUPS);
      if (ZEROS) k.zero[t] = *reinterpret_cast<const Few<uint8_t, GROUPS> *>(a.zeros + (at * 16 + r) * GROUPS);
    }
    if constexpr (FOUR) {
      const int i = b * kBlockIn;
      k.x[0][0] = i + 32 * (r / 4) < a.n_in ? *reinterpret_cast<const half8 *>(row[0] + i) : none;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = b * kBlockIn + 32 * j;
#pragma unroll
        for (int f = 0; f < MF; ++f) k.x[f][j] = i < a.n_in ? *reinterpret_cast<const half8 *>(row[f] + i) : none;
      }
    }
  };
#pragma unroll
  for (int i = 0; i < DEPTH; ++i)
    if (first + wave + i * WAVES < last) load(in[i], first + wave + i * WAVES);
  for (int b0 = first + wave; b0 < last; b0 += WAVES * DEPTH) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      const int b = b0 + i * WAVES;
      if (b >= last) break;
      const Block &k = in[i];
      half8 turned[FOUR ? 4 : 1];
      if constexpr (FOUR) {
        turned[0] = k.x[0][0];
        turned[1] = turn<12>(k.x[0][0]);
        turned[2] = turn<8>(k.x[0][0]);
        turned[3] = turn<4>(k.x[0][0]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          half2v near = {(_Float16)-1032.f, (_Float16)-1032.f}, far = {(_Float16)-72.f, (_Float16)-72.f};
          if (ZEROS) {
            near = __builtin_bit_cast(half2v, 0xe400e400u + k.zero[t].v[g] * 0x00010001u);
            far = __builtin_bit_cast(half2v, 0xd400d400u + k.zero[t].v[g] * 0x00100010u);
          }
          floatx4 part[MF] = {};
#pragma unroll
          for (int j = g * (4 / GROUPS); j < (g + 1) * (4 / GROUPS); ++j) {
            uint32_t w = k.w[t][j];
            if (kApart && g == 0) asm volatile("" : "+v"(w));
            const half8 v = unpack4bit(w, near, far);
#pragma unroll
            for (int f = 0; f < MF; ++f) part[f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, FOUR ? turned[FOUR ? j : 0] : k.x[f][FOUR ? 0 : j], part[f], 0, 0, 0);
          }
          const uint32_t s0 = k.scale[t].v[g][0], s1 = k.scale[t].v[g][1];
          const half2v lo = __builtin_bit_cast(half2v, s0), hi = __builtin_bit_cast(half2v, s1);
#pragma unroll
          for (int f = 0; f < MF; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[f][t][e] = fmaf(part[f][e], (float)(e < 2 ? lo[e & 1] : hi[e & 1]), sum[f][t][e]);
          if (kApart && g == GROUPS - 1)
#pragma unroll
            for (int f = 0; f < MF; ++f) asm volatile("" : "+v"(sum[f][t]));
        }
      if (b + WAVES * DEPTH < last) load(in[i], b + WAVES * DEPTH);
    }
  }
#pragma unroll
  for (int f = 0; f < MF; ++f)
#pragma unroll
    for (int t = 0; t < NT; ++t) shares[wave][f * NT + t][lane] = sum[f][t];
  __syncthreads();
  // 4 consecutive features of a row per thread
#pragma unroll 1
  for (int i = threadIdx.x; i < MF * NT * 64; i += 64 * WAVES) {
    const int frag = i >> 6, l = i & 63, f = frag / NT, t = frag - f * NT;
    floatx4 y = shares[0][frag][l];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) y += shares[w][frag][l];
    const int m = row0 + 16 * f + l % 16, n = (tile0 + t) * 16 + 4 * (l / 16);
    if (m >= a.m || n >= a.n_out) continue;
    if (a.cuts > 1) *reinterpret_cast<floatx4 *>(a.shares + ((int64_t)blockIdx.y * a.m + m) * a.n_out + n) = y;
    else finish(a, y, m, n);
  }
}

// Adds the cuts' shares in order
__global__ void __launch_bounds__(256) add_shares4_kernel(Linear4Args a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, size = (int64_t)a.m * a.n_out;
  if (4 * i >= size) return;
  floatx4 y = *reinterpret_cast<const floatx4 *>(a.shares + 4 * i);
  int c = 1;
  for (; c + 4 <= a.cuts; c += 4) {
    floatx4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const floatx4 *>(a.shares + (c + j) * size + 4 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) y += x[j];
  }
  for (; c < a.cuts; ++c) y += *reinterpret_cast<const floatx4 *>(a.shares + c * size + 4 * i);
  finish(a, y, (int)(4 * i / a.n_out), (int)(4 * i % a.n_out));
}

// ---- packing ----------------------------------------------------------------------------------------

struct Packed {
  uint32_t *codes;
  _Float16 *scales;
  uint8_t *zeros;
};

// What a thread writes: one 32-bit word, 8 inputs of a feature; codes(n, k) are those of inputs k .. k + 7, a byte each
template <class Codes>
__device__ __forceinline__ uint32_t pack_word(const int64_t i, const int blocks, const int n_in, const Codes &codes) {
  const int64_t block = i >> 8;
  const int lane = (i >> 2) & 63, j = i & 3, n = (int)(block / blocks) * 16 + lane % 16;
  const int k = (int)(block % blocks) * kBlockIn + 32 * j + 8 * (lane / 16);
  if (k >= n_in) return 0;
  const uint64_t c = codes(n, k);
  uint32_t w = 0;
#pragma unroll
  for (int p = 0; p < 4; ++p) w |= (uint32_t)(c >> (16 * p) & 15u) << (4 * p) | (uint32_t)(c >> (16 * p + 8) & 15u) << (16 + 4 * p);
  return w;
}

// Where the scale and the zero of feature n's group g are: `padded` groups in all, `per` in a block
__device__ __forceinline__ int64_t scale_at(const int n, const int g, const int padded, const int per) {
  return (((int64_t)(n / 16) * (padded / per) + g / per) * 4 + n % 16 / 4) * 4 * per + g % per * 4 + n % 4;
}
__device__ __forceinline__ int64_t zero_at(const int n, const int g, const int padded, const int per) {
  return (((int64_t)(n / 16) * (padded / per) + g / per) * 16 + n % 16) * per + g % per;
}

__global__ void __launch_bounds__(256) pack4_kernel(Packed to, const uint8_t *codes, int per_byte, const _Float16 *scales, const uint8_t *zeros, int n_out,
                                                    int n_in, int group) {
  const int blocks = (n_in + kBlockIn - 1) / kBlockIn, groups = n_in / group, padded = blocks * (kBlockIn / group);
  const int64_t words = (int64_t)n_out / 16 * blocks * 256, all = (int64_t)n_out * padded;
  const int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t i = i0; i < words; i += step)
    to.codes[i] = pack_word(i, blocks, n_in, [&](int n, int k) -> uint64_t {
      const int64_t at = (int64_t)n * n_in + k;
      if (per_byte == 1) return *reinterpret_cast<const uint64_t *>(codes + at);
      const uint32_t two = *reinterpret_cast<const uint32_t *>(codes + (at >> 1));
      uint64_t c = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) c |= (uint64_t)(two >> (4 * e) & 15u) << (8 * e);
      return c;
    });
  for (int64_t i = i0; i < all; i += step) {
    const int n = (int)(i / padded), g = (int)(i % padded);
    to.scales[scale_at(n, g, padded, kBlockIn / group)] = g < groups ? scales[(int64_t)n * groups + g] : (_Float16)0.f;
    if (to.zeros) to.zeros[zero_at(n, g, padded, kBlockIn / group)] = g < groups ? zeros[(int64_t)n * groups + g] & 15u : 8;
  }
}

// The scale and zero point of every group (a thread each)
__global__ void __launch_bounds__(256) scales4_kernel(Packed to, const _Float16 *src, int n_out, int n_in, int group) {
  const int blocks = (n_in + kBlockIn - 1) / kBlockIn, groups = n_in / group, padded = blocks * (kBlockIn / group);
  const int64_t all = (int64_t)n_out * padded;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int n = (int)(i / padded), g = (int)(i % padded);
    float lo = 0.f, hi = 0.f;
    bool finite = true;                  // (the minimum and the maximum pass over NaN)
    if (g < groups)
      for (int k = 0; k < group; k += 8) {
        const half8 w = *reinterpret_cast<const half8 *>(src + (int64_t)n * n_in + (int64_t)g * group + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) lo = fminf(lo, (float)w[e]), hi = fmaxf(hi, (float)w[e]), finite = finite && __builtin_isfinite((float)w[e]);
      }
    const _Float16 scale = (_Float16)(!finite ? __builtin_nanf("") : to.zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f);
    to.scales[scale_at(n, g, padded, kBlockIn / group)] = scale;
    if (to.zeros) to.zeros[zero_at(n, g, padded, kBlockIn / group)] = (float)scale > 0.f ? (uint8_t)fminf(__builtin_rintf(-lo / (float)scale), 15.f) : 8;
  }
}
__global__ void __launch_bounds__(256) codes4_kernel(Packed to, const _Float16 *src, int n_out, int n_in, int group) {
  const int blocks = (n_in + kBlockIn - 1) / kBlockIn, padded = blocks * (kBlockIn / group);
  const int64_t words = (int64_t)n_out / 16 * blocks * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256)
    to.codes[i] = pack_word(i, blocks, n_in, [&](int n, int k) -> uint64_t {
      const int g = k / group, per = kBlockIn / group;
      const float scale = (float)to.scales[scale_at(n, g, padded, per)], zero = to.zeros ? (float)to.zeros[zero_at(n, g, padded, per)] : 8.f;
      const half8 w = *reinterpret_cast<const half8 *>(src + (int64_t)n * n_in + k);
      uint64_t c = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = scale > 0.f ? __builtin_rintf((float)w[e] / scale) : 0.f;
        c |= (uint64_t)(uint32_t)fminf(fmaxf(q + zero, 0.f), 15.f) << (8 * e);
      }
      return c;
    });
}

// ---- host -------------------------------------------------------------------------------------------

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

const char *shape_problem(int32_t n_out, int32_t n_in, int32_t group) {
  if (n_out < 16 || n_out % 16 || n_out > 1 << 24) return "n_out must be a multiple of 16, at most 2^24";
  if (group != 32 && group != 64 && group != 128) return "group must be 32, 64 or 128";
  if (n_in < 32 || n_in % 32 || n_in % group || n_in > 1 << 24) return "n_in must be a multiple of 32 and of group, at most 2^24";
  return nullptr;
}

struct PackedLayout {
  int64_t blocks, scales, zeros, bytes;  // blocks of 128 inputs; byte offsets
};
PackedLayout layout_of(int32_t n_out, int32_t n_in, int32_t group, bool zeros) {
  PackedLayout l;
  l.blocks = (n_in + kBlockIn - 1) / kBlockIn;
  const int64_t groups = (int64_t)n_out * l.blocks * (kBlockIn / group);
  l.scales = (int64_t)n_out / 16 * l.blocks * 1024;
  l.zeros = l.scales + 2 * groups;
  l.bytes = l.zeros + (zeros ? groups : 0);
  return l;
}
Packed packed_at(void *p, const PackedLayout &l, bool zeros) {
  char *c = static_cast<char *>(p);
  return {reinterpret_cast<uint32_t *>(c), reinterpret_cast<_Float16 *>(c + l.scales), zeros ? reinterpret_cast<uint8_t *>(c + l.zeros) : nullptr};
}

int hip_result(const char *who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? OKV_OK : report(OKV_EHIP, "%s: %s", who, hipGetErrorString(e));
}

template <int MF, int NT, int WAVES, int DEPTH, bool FOUR = false>
void launch(const Linear4Args &a, int group, hipStream_t stream) {
  const dim3 grid((unsigned)((a.n_out / 16 + NT - 1) / NT), (unsigned)a.cuts, (unsigned)((a.m + 16 * MF - 1) / (16 * MF))), block(64 * WAVES);
  if (a.zeros) {
    if (group == 128) hipLaunchKernelGGL((linear4_kernel<MF, NT, WAVES, DEPTH, FOUR, 1, true>), grid, block, 0, stream, a);
    else if (group == 64) hipLaunchKernelGGL((linear4_kernel<MF, NT, WAVES, DEPTH, FOUR, 2, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((linear4_kernel<MF, NT, WAVES, DEPTH, FOUR, 4, true>), grid, block, 0, stream, a);
  } else {
    if (group == 128) hipLaunchKernelGGL((linear4_kernel<MF, NT, WAVES, DEPTH, FOUR, 1, false>), grid, block, 0, stream, a);
    else if (group == 64) hipLaunchKernelGGL((linear4_kernel<MF, NT, WAVES, DEPTH, FOUR, 2, false>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((linear4_kernel<MF, NT, WAVES, DEPTH, FOUR, 4, false>), grid, block, 0, stream, a);
  }
}

// Tiles of a workgroup and cuts of the inputs, by a model of the time (us, as measured with codes from HBM; what is the same for all choices
// left out).  A block of 128 inputs takes a workgroup 0.057 for each tile (0.080 of more than four with 5 to 16 rows), and 0.022 + 0.0035 a row
// (0.0070 from the 17th on) for the rows, which it fetches through L2 whatever its tiles; up to 4 rows, 0.0615, 0.1125, 0.181 and 0.256 in all
// for 1 to 4 tiles and 0.090 each of more.  One workgroup per compute unit at a time.  Cuts cost a second launch, 2.2 (3.4 with up to 16 rows) and 1.0 for each MB of
// shares.  More tiles mean fewer fetches of the rows, cuts fill the compute units again.  us, tiles x cuts: 32 rows x 4096 x 4096 4 x 4 10.0,
// 1 x 1 11.5; 32 x 4096 x 16384 8 x 8 18.8, 1 x 1 34; 128 x 12288 x 4096 6 x 1 26.7, 3 x 1 43.
struct Choice {
  int tiles, cuts;
};
Choice choose(int32_t m, int32_t n_out, int32_t n_in, int64_t workspace_bytes) {
  constexpr int kTiles[] = {1, 2, 3, 4, 6, 8}, kCuts[] = {1, 2, 3, 4, 6, 8};
  constexpr int kUnits = 256;
  const int n_tiles = n_out / 16, blocks = (n_in + kBlockIn - 1) / kBlockIn, row_groups = (m + 63) / 64, rows = std::min(m, 64);
  const double per_rows = 0.022 + 0.0035 * std::min(rows, 16) + 0.0070 * std::max(0, rows - 16);
  Choice best = {1, 1};
  double best_us = 1e30;
  for (const int t : kTiles)
    for (const int c : kCuts) {
      const double share_mb = 4e-6 * c * m * n_out;
      if (c > 1 && (blocks < 4 * c || (int64_t)c * m * n_out * 4 > workspace_bytes)) break;
      const int64_t groups = (int64_t)((n_tiles + t - 1) / t) * c * row_groups;
      const double per_block = m <= 4 ? (t == 1 ? 0.0615 : t == 2 ? 0.1125 : t == 3 ? 0.181 : t == 4 ? 0.256 : 0.090 * t)
                                      : (t > 4 && m <= 16 ? 0.080 : 0.057) * t + per_rows;
      const double us = (double)((groups + kUnits - 1) / kUnits) * ((blocks + c - 1) / c) * per_block + (c > 1 ? (m <= 16 ? 3.4 : 2.2) + share_mb : 0.0);
      if (us < best_us) best_us = us, best = {t, c};
    }
  return best;
}

}  // namespace

}  // namespace okv

using namespace okv;

extern "C" {

int64_t okv_linear4_packed_bytes(int32_t n_out, int32_t n_in, int32_t group, int32_t zeros) {
  if (const char *why = shape_problem(n_out, n_in, group)) return report(OKV_EINVAL, "okv_linear4_packed_bytes: %s", why);
  return layout_of(n_out, n_in, group, zeros != 0).bytes;
}

int okv_linear4_pack(void *dst, const void *codes, int32_t per_byte, const void *scales, const void *zeros, int32_t n_out, int32_t n_in, int32_t group,
                     void *stream) {
  if (const char *why = shape_problem(n_out, n_in, group)) return report(OKV_EINVAL, "okv_linear4_pack: %s", why);
  if (!dst || !codes || !scales || !aligned16(dst) || !aligned16(codes)) return report(OKV_EINVAL, "okv_linear4_pack: NULL or misaligned pointer");
  if (per_byte != 1 && per_byte != 2) return report(OKV_EINVAL, "okv_linear4_pack: per_byte must be 1 or 2");
  const PackedLayout l = layout_of(n_out, n_in, group, zeros != nullptr);
  const int64_t words = (int64_t)n_out / 16 * l.blocks * 256;
  hipLaunchKernelGGL(pack4_kernel, dim3((unsigned)std::min<int64_t>((words + 255) / 256, 1 << 14)), dim3(256), 0, static_cast<hipStream_t>(stream),
                     packed_at(dst, l, zeros != nullptr), static_cast<const uint8_t *>(codes), per_byte, static_cast<const _Float16 *>(scales),
                     static_cast<const uint8_t *>(zeros), n_out, n_in, group);
  return hip_result("okv_linear4_pack");
}

int okv_linear4_quantize(void *dst, const void *src, int32_t n_out, int32_t n_in, int32_t group, int32_t zeros, void *stream) {
  if (const char *why = shape_problem(n_out, n_in, group)) return report(OKV_EINVAL, "okv_linear4_quantize: %s", why);
  if (!dst || !src || !aligned16(dst) || !aligned16(src)) return report(OKV_EINVAL, "okv_linear4_quantize: NULL or misaligned pointer");
  const PackedLayout l = layout_of(n_out, n_in, group, zeros != 0);
  const Packed to = packed_at(dst, l, zeros != 0);
  const int64_t words = (int64_t)n_out / 16 * l.blocks * 256, groups = (int64_t)n_out * l.blocks * (kBlockIn / group);
  hipLaunchKernelGGL(scales4_kernel, dim3((unsigned)std::min<int64_t>((groups + 255) / 256, 1 << 14)), dim3(256), 0, static_cast<hipStream_t>(stream), to,
                     static_cast<const _Float16 *>(src), n_out, n_in, group);
  hipLaunchKernelGGL(codes4_kernel, dim3((unsigned)std::min<int64_t>((words + 255) / 256, 1 << 14)), dim3(256), 0, static_cast<hipStream_t>(stream), to,
                     static_cast<const _Float16 *>(src), n_out, n_in, group);
  return hip_result("okv_linear4_quantize");
}

int64_t okv_linear4_workspace_bytes(int32_t m, int32_t n_out, int32_t n_in) {
  if (const char *why = shape_problem(n_out, n_in, 32)) return report(OKV_EINVAL, "okv_linear4_workspace_bytes: %s", why);
  if (m < 1 || m > OKV_LINEAR4_MAX_BATCH) return report(OKV_EINVAL, "okv_linear4_workspace_bytes: m must be in [1, %d]", OKV_LINEAR4_MAX_BATCH);
  const Choice c = choose(m, n_out, n_in, INT64_MAX);
  return c.cuts > 1 ? (int64_t)c.cuts * m * n_out * 4 : 0;
}

int okv_linear4(const void *x, const void *packed, const void *bias, const void *residual, void *const *out, const int32_t *cols, int32_t n_seg, int32_t m,
                int32_t n_out, int32_t n_in, int32_t group, int32_t zeros, int32_t relu, void *workspace, int64_t workspace_bytes, void *stream) {
  if (const char *why = shape_problem(n_out, n_in, group)) return report(OKV_EINVAL, "okv_linear4: %s", why);
  if (m < 1 || m > OKV_LINEAR4_MAX_BATCH) return report(OKV_EINVAL, "okv_linear4: m must be in [1, %d]", OKV_LINEAR4_MAX_BATCH);
  if (!x || !packed || !out) return report(OKV_EINVAL, "okv_linear4: NULL pointer");
  if (!aligned16(x) || !aligned16(packed) || !aligned16(bias) || !aligned16(residual)) return report(OKV_EINVAL, "okv_linear4: misaligned pointer");
  if (n_seg < 1 || n_seg > 3) return report(OKV_EINVAL, "okv_linear4: n_seg must be 1, 2 or 3");
  if (residual && n_seg != 1) return report(OKV_EINVAL, "okv_linear4: a residual goes with one output tensor");
  Linear4Args a;
  int64_t end = 0;
  for (int s = 0; s < 3; ++s) {
    if (s < n_seg) {
      const int64_t width = cols ? cols[s] : n_out / n_seg;
      if (width < 16 || width % 16) return report(OKV_EINVAL, "okv_linear4: the runs of output features must be multiples of 16");
      if (!out[s] || !aligned16(out[s])) return report(OKV_EINVAL, "okv_linear4: NULL or misaligned output");
      end += width;
    }
    a.out[s] = static_cast<_Float16 *>(out[std::min(s, n_seg - 1)]);
    a.end[s] = (int32_t)std::min<int64_t>(end, 0x7fffffff);
  }
  if (end != n_out) return report(OKV_EINVAL, "okv_linear4: the runs of output features must add up to n_out");
  const PackedLayout l = layout_of(n_out, n_in, group, zeros != 0);
  const Packed p = packed_at(const_cast<void *>(packed), l, zeros != 0);
  a.x = static_cast<const _Float16 *>(x);
  a.codes = reinterpret_cast<const u32x4 *>(p.codes), a.scales = p.scales, a.zeros = p.zeros;
  a.bias = static_cast<const _Float16 *>(bias), a.residual = static_cast<const _Float16 *>(residual);
  a.m = m, a.n_out = n_out, a.n_in = n_in, a.blocks = (int32_t)l.blocks, a.relu = relu != 0;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const Choice c = choose(m, n_out, n_in, workspace && aligned16(workspace) ? workspace_bytes : 0);
  a.cuts = c.cuts, a.shares = static_cast<float *>(workspace);
  // wavefronts and blocks in flight of each: as measured for 16, 32 and 64 rows (registers bound both)
  if (m <= 4) {
    switch (c.tiles) {
      case 1: launch<1, 1, 16, 2, true>(a, group, st); break;
      case 2: launch<1, 2, 8, 1, true>(a, group, st); break;
      case 3: launch<1, 3, 16, 1, true>(a, group, st); break;
      case 4: launch<1, 4, 16, 1, true>(a, group, st); break;
      case 6: launch<1, 6, 8, 1, true>(a, group, st); break;
      default: launch<1, 8, 8, 1, true>(a, group, st); break;
    }
  } else if (m <= 16) {
    switch (c.tiles) {
      case 1: launch<1, 1, 16, 2>(a, group, st); break;
      case 2: launch<1, 2, 8, 2>(a, group, st); break;
      case 3: launch<1, 3, 16, 1>(a, group, st); break;
      case 4: launch<1, 4, 16, 1>(a, group, st); break;
      case 6: launch<1, 6, 8, 1>(a, group, st); break;
      default: launch<1, 8, 8, 1>(a, group, st); break;
    }
  } else if (m <= 32) {
    switch (c.tiles) {
      case 1: launch<2, 1, 8, 2>(a, group, st); break;
      case 2: launch<2, 2, 8, 2>(a, group, st); break;
      case 3: launch<2, 3, 8, 1>(a, group, st); break;
      case 4: launch<2, 4, 8, 1>(a, group, st); break;
      case 6: launch<2, 6, 8, 1>(a, group, st); break;
      default: launch<2, 8, 8, 1>(a, group, st); break;
    }
  } else {
    switch (c.tiles) {
      case 1: launch<4, 1, 8, 1>(a, group, st); break;
      case 2: launch<4, 2, 8, 1>(a, group, st); break;
      case 3: launch<4, 3, 8, 1>(a, group, st); break;
      case 4: launch<4, 4, 4, 1>(a, group, st); break;
      case 6: launch<4, 6, 4, 1>(a, group, st); break;
      default: launch<4, 8, 4, 1>(a, group, st); break;
    }
  }
  if (a.cuts > 1) hipLaunchKernelGGL(add_shares4_kernel, dim3((unsigned)(((int64_t)m * n_out / 4 + 255) / 256)), dim3(256), 0, st, a);
  return hip_result("okv_linear4");
}

}  // extern "C"
