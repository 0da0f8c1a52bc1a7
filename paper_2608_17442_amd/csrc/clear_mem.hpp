// Global memory as the kernels of the block in the clear see it: a base that
// is the same for a wave, and byte offsets below 2^31 from it.  An access at
// kAbsent reads zero and writes nothing, so that edges need no branches, which
// would hold back the loads behind them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace fesc {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr uint32_t kAbsent = 0xfffffff0u;

template <typename T>
__device__ __forceinline__ auto to_four(const f32x4& v) {
  if constexpr (sizeof(T) == 4)
    return v;
  else
    return __builtin_convertvector(v, bf16x4);
}

struct Mem {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ explicit Mem(const void* base)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, 0x7fffffff, 0x00027000)) {}
  __device__ __forceinline__ u32x4 load16(uint32_t at) const {
    return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
  }
  __device__ __forceinline__ void store16(uint32_t at, const u32x4& v) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, r, at, 0, 0);
  }
  template <typename T>
  __device__ __forceinline__ uint32_t load_bits(uint32_t at) const {
    if constexpr (sizeof(T) == 4)
      return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
    else
      return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
  }
  template <typename T>
  __device__ __forceinline__ void store_bits(uint32_t at, uint32_t v) const {
    if constexpr (sizeof(T) == 4)
      __builtin_amdgcn_raw_buffer_store_b32(v, r, at, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b16((short)v, r, at, 0, 0);
  }
  template <typename T>
  __device__ __forceinline__ static float value(uint32_t bits) {
    return __uint_as_float(sizeof(T) == 4 ? bits : bits << 16);
  }
  template <typename T>
  __device__ __forceinline__ float load(uint32_t at) const {
    return value<T>(load_bits<T>(at));
  }
  // Four neighbouring elements at byte offset `at`, those at or past `left`
  // absent; WHOLE: all or none, in one access.
  template <typename T, bool WHOLE>
  __device__ __forceinline__ void store_four(uint32_t at, const f32x4& v, int left) const {
    const auto o = to_four<T>(v);
    if constexpr (WHOLE) {
      if constexpr (sizeof(T) == 4)
        store16(left > 0 ? at : kAbsent, __builtin_bit_cast(u32x4, o));
      else
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, o), r,
                                              left > 0 ? at : kAbsent, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t to = i < left ? at + i * (uint32_t)sizeof(T) : kAbsent;
        if constexpr (sizeof(T) == 4)
          store_bits<T>(to, __float_as_uint(o[i]));
        else
          store_bits<T>(to, (uint16_t)__builtin_bit_cast(s16x4, o)[i]);
      }
    }
  }
  template <bool WHOLE>
  __device__ __forceinline__ f32x4 load_four(uint32_t at, int left) const {
    if constexpr (WHOLE) return __builtin_bit_cast(f32x4, load16(left > 0 ? at : kAbsent));
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = load<float>(i < left ? at + 4 * i : kAbsent);
    return v;
  }
};

// Sums over the 16 lanes of a row without leaving the registers, and over the
// lanes l, l ^ 16, l ^ 32, l ^ 48.
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
  return __uint_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float v) {
  v += dpp_move<0xb1>(v);   // quad_perm 1 0 3 2
  v += dpp_move<0x4e>(v);   // quad_perm 2 3 0 1
  v += dpp_move<0x141>(v);  // row_half_mirror
  v += dpp_move<0x140>(v);  // row_mirror
  return v;
}
// Sixteen such sums at once: lane l % 16 gets that of v[l % 16].  Each step
// halves the values and hands the others to a lane that keeps them.
__device__ __forceinline__ float sums16(float (&v)[16]) {
  const int l = threadIdx.x & 15;
  auto halve = [&](auto n, bool upper, auto move) {
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float a = v[i], b = v[i + n];
      v[i] = (upper ? b : a) + move(upper ? a : b);
    }
  };
  halve(std::integral_constant<int, 8>{}, l & 8, [](float x) { return dpp_move<0x140>(x); });
  halve(std::integral_constant<int, 4>{}, l & 4, [](float x) { return dpp_move<0x141>(x); });
  halve(std::integral_constant<int, 2>{}, l & 2, [](float x) { return dpp_move<0x4e>(x); });
  halve(std::integral_constant<int, 1>{}, l & 1, [](float x) { return dpp_move<0xb1>(x); });
  return v[0];
}
// A column of four rows in each of the groups l / 16, v already summed from its rows on
// within a group: adds the groups that follow, and `below`.  Returns the whole sum.
__device__ __forceinline__ float add_later_groups(f32x4& v, float below) {
  const int g = (threadIdx.x & 63) >> 4;
  const float next = __shfl_xor(v[0], 16);
  const float both = v[0] + next, far = __shfl_xor(both, 32);
  const float more = below + ((g & 1 ? 0.0f : next) + (g & 2 ? 0.0f : far));
  const float whole = below + (both + far);
  v += more;
  return whole;
}
__device__ __forceinline__ float sum_groups(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

}  // namespace fesc
