// Exchanges and reductions inside a wavefront of 64 lanes (device code, gfx950).
#pragma once

#include <hip/hip_runtime.h>

namespace okv {

// Values of other lanes of a wavefront without the round trip through LDS that a shuffle is (some 50 ns, one after the other in
// every chain below).  The swaps exchange the odd rows of 16 lanes (the upper half of the wavefront) of one register with the even rows
// (the lower half) of another: of two copies of a value one then holds lane & ~16 (& ~32) of it in every lane, the other lane | 16 (| 32).
// Written as assembly: the compiler's builtin returned the first register twice.
// us, shuffles -> these: a layer of 32 sequences x 768 keys x 32 heads (d = 128) 61.2 -> 59.9, 16 ragged sequences of 32 heads with
// their joining launch 35.5 -> 33.5, a step of 4 layers of two long sequences of 32 / 8 heads 57 -> 55.5.
template <int X>
__device__ __forceinline__ void split_lanes(const float v, float &a, float &b) {
  static_assert(X == 16 || X == 32, "");
  a = v, b = v;
  if constexpr (X == 16) asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  else asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
}
template <int X>
__device__ __forceinline__ float max_with_lane_xor(const float v) {
  float a, b;
  split_lanes<X>(v, a, b);
  return fmaxf(a, b);
}
template <int X>
__device__ __forceinline__ float sum_with_lane_xor(const float v) {
  float a, b;
  split_lanes<X>(v, a, b);
  return a + b;
}
// the value CTRL lanes further in the row of 16 (row_ror: CTRL - 0x120)
template <int CTRL>
__device__ __forceinline__ float row_turned(const float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
// Over all 64 lanes, which all take part, in the order of a butterfly from lane ^ 32 to lane ^ 1 (a value that repeats every 2 n lanes is
// the same n lanes further as in lane ^ n)
__device__ __forceinline__ float wave_max(float v) {
  v = max_with_lane_xor<16>(max_with_lane_xor<32>(v));
  v = fmaxf(v, row_turned<0x128>(v));
  v = fmaxf(v, row_turned<0x124>(v));
  v = fmaxf(v, row_turned<0x122>(v));
  return fmaxf(v, row_turned<0x121>(v));
}
__device__ __forceinline__ float row_sum(float v) {      // over the lane's row of 16
  v += row_turned<0x128>(v);
  v += row_turned<0x124>(v);
  v += row_turned<0x122>(v);
  return v + row_turned<0x121>(v);
}
__device__ __forceinline__ float wave_sum(float v) { return row_sum(sum_with_lane_xor<16>(sum_with_lane_xor<32>(v))); }

// The value that DPP control CTRL brings to each lane, 0 where it brings none; ROWS: the rows of 16 lanes that take it
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int brought(const int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t brought(const uint64_t v) { return (uint64_t)(uint32_t)brought<CTRL, ROWS>((int)(v >> 32)) << 32 | (uint32_t)brought<CTRL, ROWS>((int)v); }
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double brought(const double v) { return __builtin_bit_cast(double, brought<CTRL, ROWS>(__builtin_bit_cast(uint64_t, v))); }
// Sums over the lanes up to each one, itself included: within rows of 16 (lanes 1, 2, 4 and 8 before), then the last lane of a row on to the next row, and lane 31 to the upper half
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
  v += brought<0x111>(v);
  v += brought<0x112>(v);
  v += brought<0x114>(v);
  v += brought<0x118>(v);
  v += brought<0x142, 0xa>(v);
  return v + brought<0x143, 0xc>(v);
}
// Lane `from`'s value, in scalar registers
__device__ __forceinline__ int lane_value(const int v, const int from) { return __builtin_amdgcn_readlane(v, from); }
__device__ __forceinline__ uint64_t lane_value(const uint64_t v, const int from) { return (uint64_t)(uint32_t)lane_value((int)(v >> 32), from) << 32 | (uint32_t)lane_value((int)v, from); }
__device__ __forceinline__ double lane_value(const double v, const int from) { return __builtin_bit_cast(double, lane_value(__builtin_bit_cast(uint64_t, v), from)); }
__device__ __forceinline__ double wave_sum(const double v) { return lane_value(wave_scan(v), 63); }

}  // namespace okv
