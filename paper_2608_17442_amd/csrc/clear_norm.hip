// The norms of the block in the clear, fused with what stands before them:
//   gated     v = (m + skip x) silu(z),  u = v k w      (after the recurrence)
//   residual  v = r + scale o,           u = v k w      (before the next block; v is
//                                                       returned too)
// k = 1 / sqrt(mean v^2 + eps) over a row of `width` channels.  With g = du w,
//   dv = k (g - v k^2 mean(g v))   (+ the gradient that reaches v itself)
//   dw = sum over rows of du v k
// Everything is fp32 between the loads and the stores.  All kernels are bound
// by memory: each array passes once, a row staying in the registers of the
// lanes that share it, for the gradient too (v is formed again from its
// inputs rather than kept).
// 16384 rows of 1536 in bfloat16, gated: 31 us (201 MB, 6.5 TB/s, in part from the
// memory-side cache), gradient 58 + 4 us (352 MB, 5.7 TB/s); of 768, residual: 17 us,
// gradient 25 + 4.
#include <type_traits>

#include "clear.hpp"
#include "clear_mem.hpp"
#include "fesc_internal.hpp"

namespace fesc {

namespace {

constexpr int kUnit = 8;       // channels of one lane's unit
constexpr int kThreads = 256;

// Eight channels as they lie in memory.  VEC (rows start at multiples of 16
// bytes and hold whole units): neighbours.  Otherwise STEP apart, so that the
// lanes of a wave read neighbours.  Those at or past `left` are zero.
template <typename T, bool VEC, int LANES>
struct Unit {
  static constexpr int STEP = VEC ? 1 : LANES;
  // first channel of unit j of a lane
  __device__ __forceinline__ static int channel(int lane, int j) {
    return VEC ? (lane + j * LANES) * kUnit : lane + j * LANES * kUnit;
  }
  static constexpr int kWords = kUnit * sizeof(T) / 4;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const Mem& m, int channel, int left) {
    const uint32_t at = channel * (uint32_t)sizeof(T);
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const u32x4 v = m.load16(left > 0 ? at + 4 * i : kAbsent);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i + j] = v[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        const uint32_t v = m.load_bits<T>(i * STEP < left ? at + i * STEP * (uint32_t)sizeof(T) : kAbsent);
        if constexpr (sizeof(T) == 4)
          w[i] = v;
        else
          w[i / 2] |= v << (16 * (i & 1));
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(w[i]);
    else
      return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set(int i, const f32x4& v) {  // channels i .. i + 3
    const auto o = to_four<T>(v);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = __float_as_uint(o[j]);
    } else {
      const u32x2 p = __builtin_bit_cast(u32x2, o);
      w[i / 2] = p[0];
      w[i / 2 + 1] = p[1];
    }
  }
  __device__ __forceinline__ void store(const Mem& m, int channel, int left) const {
    const uint32_t at = channel * (uint32_t)sizeof(T);
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        m.store16(left > 0 ? at + 4 * i : kAbsent, u32x4{w[i], w[i + 1], w[i + 2], w[i + 3]});
    } else {
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        m.store_bits<T>(i * STEP < left ? at + i * STEP * (uint32_t)sizeof(T) : kAbsent,
                        sizeof(T) == 4 ? w[i] : w[i / 2] >> (16 * (i & 1)) & 0xffffu);
    }
  }
};

// Sums over the TPR lanes that share a row: in a wave, then over its waves
// through LDS.
template <int TPR, typename V>
__device__ __forceinline__ V row_sum(V v, V* red) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    v.x += __shfl_xor(v.x, d);
    v.y += __shfl_xor(v.y, d);
  }
  if constexpr (TPR > 64) {
    constexpr int kWaves = TPR / 64;
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    const V* r = red + wave / kWaves * kWaves;
    v = r[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) {
      v.x += r[i].x;
      v.y += r[i].y;
    }
  }
  return v;
}

// 1 / (1 + e^{-z}) from the hardware's base-2 exponential and reciprocal: off
// by a few units of the last place of fp32 for z >= 0; below, where the result
// nears e^{z}, by some 2^-24 |z| of it, and it is 0 below about -88.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

// The row of this wave among those that the workgroup holds at once, and the
// same for every lane of it.
template <int TPR>
__device__ __forceinline__ uint32_t own_row() {
  return __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
}

// A row is shared by TPR lanes, UPT units each.
template <typename T, bool GATED, int TPR, int UPT, bool VEC>
__global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
  __shared__ float2 red[kThreads / 64];
  constexpr int kRows = kThreads / TPR;
  const int lane = threadIdx.x % TPR;
  Unit<T, VEC, TPR> kk[UPT], ww[UPT];
  const Mem km(a.k), wm(a.w);
#pragma unroll
  for (int j = 0; j < UPT; ++j) {
    const int e = Unit<T, VEC, TPR>::channel(lane, j), left = (int)a.width - e;
    kk[j].load(km, e, left);
    ww[j].load(wm, e, left);
  }
  for (uint64_t base = (uint64_t)blockIdx.x * kRows; base < a.rows;
       base += (uint64_t)gridDim.x * kRows) {
    const uint64_t row = base + own_row<TPR>();
    const int width = row < a.rows ? a.width : 0;  // of an absent row: nothing
    const Mem ma((const T*)a.a + row * a.a_row), mb((const T*)a.b + row * a.b_row);
    const Mem mc((const T*)a.c + row * a.c_row);
    Unit<T, VEC, TPR> ua[UPT], ub[UPT], uc[UPT];
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = Unit<T, VEC, TPR>::channel(lane, j), left = width - e;
      ua[j].load(ma, e, left);
      ub[j].load(mb, e, left);
      if constexpr (GATED) uc[j].load(mc, e, left);
    }
    float v[UPT][kUnit];
    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        if constexpr (GATED) {
          const float z = uc[j].get(i);
          v[j][i] = __builtin_fmaf(kk[j].get(i), ub[j].get(i), ua[j].get(i)) * (z * sigmoid(z));
        } else {
          v[j][i] = __builtin_fmaf(kk[j].get(i), ua[j].get(i), ub[j].get(i));
        }
        sum.x = __builtin_fmaf(v[j][i], v[j][i], sum.x);
      }
    }
    sum = row_sum<TPR>(sum, red);
    const float k = 1.0f / sqrtf(sum.x / (float)a.width + a.eps);
    const Mem mu((T*)a.u + row * a.width), mr((T*)a.r_new + row * a.width);
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = Unit<T, VEC, TPR>::channel(lane, j), left = width - e;
      Unit<T, VEC, TPR> o;
      if constexpr (!GATED) {
#pragma unroll
        for (int i = 0; i < kUnit; i += 4)
          o.set(i, f32x4{v[j][i], v[j][i + 1], v[j][i + 2], v[j][i + 3]});
        o.store(mr, e, left);
      }
#pragma unroll
      for (int i = 0; i < kUnit; i += 4) {
        f32x4 u;
#pragma unroll
        for (int h = 0; h < 4; ++h) u[h] = v[j][i + h] * k * ww[j].get(i + h);
        o.set(i, u);
      }
      o.store(mu, e, left);
    }
  }
}

// Gradients.  The sums over rows (dk: skip or scale; dw) go to one fp32 row
// per workgroup, added up by k_norm_parts: no atomics, so a result does not
// depend on the order of execution.  In rows of up to 512 channels the row's
// two sums and the difference g - v k^2 mean(g v) are fp64: where g is nearly
// parallel to v, as it always is in a row of one channel, the difference is far
// smaller than its terms.
// The next row's loads are under way while a row is worked on (where a lane
// holds at most two units: more would not fit the registers).
template <typename T, bool GATED, int TPR, int UPT, bool VEC>
__global__ __launch_bounds__(kThreads) void k_norm_grad(NormArgs a) {
  constexpr bool kDouble = TPR == 64 && UPT == 1;
  constexpr bool kAhead = UPT <= 2;
  using Sum = std::conditional_t<kDouble, double, float>;
  using Sums = std::conditional_t<kDouble, double2, float2>;
  constexpr int kRows = kThreads / TPR;
  constexpr int W = TPR * UPT * kUnit;
  __shared__ Sums red[kThreads / 64];
  __shared__ float part[kRows > 1 ? 2 * W : 1];
  const int lane = threadIdx.x % TPR;
  Unit<T, VEC, TPR> kk[UPT], ww[UPT];
  float dk[UPT][kUnit], dw[UPT][kUnit];
  const Mem km(a.k), wm(a.w);
#pragma unroll
  for (int j = 0; j < UPT; ++j) {
    const int e = Unit<T, VEC, TPR>::channel(lane, j), left = (int)a.width - e;
    kk[j].load(km, e, left);
    ww[j].load(wm, e, left);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) dk[j][i] = dw[j][i] = 0.0f;
  }
  struct Row {
    Unit<T, VEC, TPR> a[UPT], b[UPT], c[UPT], du[UPT], dr[UPT];
  };
  auto fetch = [&](Row& r, uint64_t base) {
    const uint64_t row = base + own_row<TPR>();
    const int width = row < a.rows ? a.width : 0;
    const Mem ma((const T*)a.a + row * a.a_row), mb((const T*)a.b + row * a.b_row);
    const Mem mc((const T*)a.c + row * a.c_row), md((const T*)a.du + row * a.du_row);
    const Mem mr((const T*)a.dr_new + row * a.dr_row);
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = Unit<T, VEC, TPR>::channel(lane, j), left = width - e;
      r.a[j].load(ma, e, left);
      r.b[j].load(mb, e, left);
      if constexpr (GATED) r.c[j].load(mc, e, left);
      r.du[j].load(md, e, a.du ? left : 0);
      if constexpr (!GATED) r.dr[j].load(mr, e, a.dr_new ? left : 0);
    }
  };
  const uint64_t step = (uint64_t)gridDim.x * kRows;
  uint64_t base = (uint64_t)blockIdx.x * kRows;
  Row next;
  if constexpr (kAhead) fetch(next, base);
  for (; base < a.rows; base += step) {
    Row r;
    if constexpr (kAhead) {
      r = next;
      fetch(next, base + step);
    } else {
      fetch(r, base);
    }
    Sums sum = {0, 0};
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        float v;
        if constexpr (GATED) {
          const float z = r.c[j].get(i);
          v = __builtin_fmaf(kk[j].get(i), r.b[j].get(i), r.a[j].get(i)) * (z * sigmoid(z));
        } else {
          v = __builtin_fmaf(kk[j].get(i), r.a[j].get(i), r.b[j].get(i));
        }
        const float g = r.du[j].get(i) * ww[j].get(i);
        if constexpr (kDouble) {
          sum.x = __builtin_fma((double)v, (double)v, sum.x);
          sum.y = __builtin_fma((double)g, (double)v, sum.y);
        } else {
          sum.x = __builtin_fmaf(v, v, sum.x);
          sum.y = __builtin_fmaf(g, v, sum.y);
        }
      }
    }
    sum = row_sum<TPR>(sum, red);
    const Sum mean = sum.x / a.width + a.eps, c = sum.y / a.width / mean;
    const float k = 1.0f / sqrtf((float)mean);
    const uint64_t row = base + own_row<TPR>();
    const int width = row < a.rows ? a.width : 0;
    const Mem ma((T*)a.da + row * a.width), mb((T*)a.db + row * a.width);
    const Mem mc((T*)a.dc + row * a.width);
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = Unit<T, VEC, TPR>::channel(lane, j), left = width - e;
      Unit<T, VEC, TPR> o1, o2, o3;
#pragma unroll
      for (int i4 = 0; i4 < kUnit; i4 += 4) {
        f32x4 v1, v2, v3;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const int i = i4 + h;
          const float du = r.du[j].get(i), kv = kk[j].get(i), g = du * ww[j].get(i);
          auto along = [&](float v) {  // dv / k
            if constexpr (kDouble)
              return (float)__builtin_fma(-(double)v, c, (double)g);
            else
              return __builtin_fmaf(-v, c, g);
          };
          if constexpr (GATED) {
            const float z = r.c[j].get(i), sg = sigmoid(z), gate = z * sg, x = r.b[j].get(i);
            const float q = __builtin_fmaf(kv, x, r.a[j].get(i)), v = q * gate;
            const float dv = k * along(v), dq = dv * gate;
            dw[j][i] = __builtin_fmaf(du, v * k, dw[j][i]);
            dk[j][i] = __builtin_fmaf(x, dq, dk[j][i]);
            v1[h] = dq;
            v2[h] = kv * dq;
            v3[h] = dv * q * __builtin_fmaf(gate, 1.0f - sg, sg);
          } else {
            const float o = r.a[j].get(i);
            const float v = __builtin_fmaf(kv, o, r.b[j].get(i));
            const float dv = __builtin_fmaf(k, along(v), r.dr[j].get(i));
            dw[j][i] = __builtin_fmaf(du, v * k, dw[j][i]);
            dk[j][i] = __builtin_fmaf(o, dv, dk[j][i]);
            v1[h] = kv * dv;
            v2[h] = dv;
          }
        }
        o1.set(i4, v1);
        o2.set(i4, v2);
        if constexpr (GATED) o3.set(i4, v3);
      }
      o1.store(ma, e, left);
      o2.store(mb, e, left);
      if constexpr (GATED) o3.store(mc, e, left);
    }
  }
  float* out = a.part + (uint64_t)blockIdx.x * 2 * a.width;
  if constexpr (kRows > 1) {
    for (int w = 0; w < kRows; ++w) {
      if ((int)(threadIdx.x / TPR) == w) {
#pragma unroll
        for (int j = 0; j < UPT; ++j) {
#pragma unroll
          for (int i = 0; i < kUnit; ++i) {
            const int e = Unit<T, VEC, TPR>::channel(lane, j) + i * Unit<T, VEC, TPR>::STEP;
            part[e] = (w ? part[e] : 0.0f) + dk[j][i];
            part[W + e] = (w ? part[W + e] : 0.0f) + dw[j][i];
          }
        }
      }
      __syncthreads();
    }
    for (int e = threadIdx.x; e < (int)a.width; e += kThreads) {
      out[e] = part[e];
      out[a.width + e] = part[W + e];
    }
  } else {
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        const int e = Unit<T, VEC, TPR>::channel(lane, j) + i * Unit<T, VEC, TPR>::STEP;
        if (e < (int)a.width) {
          out[e] = dk[j][i];
          out[a.width + e] = dw[j][i];
        }
      }
    }
  }
}

// Column sums of the workgroups' rows: 16 columns by 16 groups of rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_parts(NormArgs a) {
  __shared__ float red[16][17];
  const int col = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const uint32_t e = blockIdx.x * 16 + col;
  float s = 0.0f;
  if (e < 2 * a.width) {
    const float* p = a.part + e;
    const uint64_t pitch = 2 * a.width;
    uint32_t r = grp;
    for (; r + 112 < a.blocks; r += 128) {  // eight loads under way at once
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[(r + 16 * k) * pitch];
      s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    for (; r < a.blocks; r += 16) s += p[r * pitch];
  }
  red[grp][col] = s;
  __syncthreads();
  if (grp == 0 && e < 2 * a.width) {
    s = 0.0f;
#pragma unroll
    for (int g = 0; g < 16; ++g) s += red[g][col];
    if (e < a.width)
      ((T*)a.dk)[e] = (T)s;
    else
      ((T*)a.dw)[e - a.width] = (T)s;
  }
}

// Lanes that share a row, by its units (unaligned rows: at least 256 lanes,
// whose loads go element by element anyway).  The gradient at 1536 channels, 16384
// rows: 128 lanes of two units, with the next row's loads under way, 59 us; 256 of
// one 122; 64 of three, without, 149.
uint32_t lanes_of(uint32_t width, bool vec) {
  const uint32_t units = (width + kUnit - 1) / kUnit;
  return units <= 64 || (units <= 128 && vec) ? 64 : units <= 256 && vec ? 128 : 256;
}

template <typename T, bool GATED, bool GRAD>
hipError_t norm(const NormArgs& a, uint32_t blocks, hipStream_t s) {
  const uint32_t units = (a.width + kUnit - 1) / kUnit;
#define RUN(TPR, UPT, VEC)                                                  \
  do {                                                                      \
    if constexpr (GRAD)                                                     \
      k_norm_grad<T, GATED, TPR, UPT, VEC><<<blocks, kThreads, 0, s>>>(a);  \
    else                                                                    \
      k_norm<T, GATED, TPR, UPT, VEC><<<blocks, kThreads, 0, s>>>(a);       \
  } while (0)
  if (a.vec) {
    if (units <= 64) RUN(64, 1, true);
    else if (units <= 128) RUN(64, 2, true);
    else if (units <= 256) RUN(128, 2, true);
    else if (units <= 512) RUN(256, 2, true);
    else if (units <= 1024) RUN(256, 4, true);
    else RUN(256, 8, true);
  } else {
    if (units <= 64) RUN(64, 1, false);
    else if (units <= 256) RUN(256, 1, false);
    else if (units <= 1024) RUN(256, 4, false);
    else RUN(256, 8, false);
  }
#undef RUN
  return hipGetLastError();
}

}  // namespace

// Workgroups of a gradient: two on a compute unit, each of which leaves a row of
// partial sums; one for wide rows, whose partial sums weigh most.  16384 rows of
// 1536, 256, 512, 1024 workgroups: 66, 60, 64 us; 4096 rows of 1536: 22.7, 21.8, 26;
// 4096 of 4096: 43, 47, 61; 4096 of 8192: 103, 116, 145.
uint32_t norm_grad_blocks(uint64_t rows, uint32_t width, bool vec) {
  const uint32_t at_once = kThreads / lanes_of(width, vec);
  const uint64_t n = (rows + at_once - 1) / at_once, most = width < 4096 ? 512 : 256;
  return (uint32_t)(n < most ? n : most);
}

hipError_t launch_norm(uint32_t dtype, bool gated, const NormArgs& a, hipStream_t s) {
  const uint32_t at_once = kThreads / lanes_of(a.width, a.vec);
  const uint64_t n = (a.rows + at_once - 1) / at_once;
  // 16384 rows of 1536: 4096 workgroups 31.8 us, 8192 30.6; 65536 of 384: 32.3, 31.5,
  // 16384 30.6
  const uint32_t blocks = (uint32_t)(n < 16384 ? n : 16384);
  if (dtype == FESC_BF16)
    return gated ? norm<__bf16, true, false>(a, blocks, s) : norm<__bf16, false, false>(a, blocks, s);
  return gated ? norm<float, true, false>(a, blocks, s) : norm<float, false, false>(a, blocks, s);
}

hipError_t launch_norm_grad(uint32_t dtype, bool gated, const NormArgs& a, hipStream_t s) {
  if (a.blocks) {
    hipError_t e;
    if (dtype == FESC_BF16)
      e = gated ? norm<__bf16, true, true>(a, a.blocks, s) : norm<__bf16, false, true>(a, a.blocks, s);
    else
      e = gated ? norm<float, true, true>(a, a.blocks, s) : norm<float, false, true>(a, a.blocks, s);
    if (e) return e;
  }
  const uint32_t grid = (2 * a.width + 15) / 16;
  if (dtype == FESC_BF16)
    k_norm_parts<__bf16><<<grid, kThreads, 0, s>>>(a);
  else
    k_norm_parts<float><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace fesc
