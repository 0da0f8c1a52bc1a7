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
#include "clear.hpp"
#include "fesc_internal.hpp"

namespace fesc {

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kUnit = 8;       // neighbouring channels of one lane
constexpr int kThreads = 256;

// Eight neighbouring channels as they lie in memory.
template <typename T>
struct Unit {
  static constexpr int kWords = kUnit * sizeof(T) / 4;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const T* p, int left, bool vec) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
    if (vec) {
      if (left > 0) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint32_t*>(p) + i);
#pragma unroll
          for (int j = 0; j < 4; ++j) w[i + j] = v[j];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        if (i < left) {
          if constexpr (sizeof(T) == 4)
            w[i] = *reinterpret_cast<const uint32_t*>(p + i);
          else
            w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + i) << (16 * (i & 1));
        }
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(w[i]);
    else
      return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

template <typename T>
__device__ __forceinline__ void store_unit(T* p, const float* v, int left, bool vec) {
  T t[kUnit];
#pragma unroll
  for (int i = 0; i < kUnit; ++i) t[i] = (T)v[i];
  if (vec) {
    if (left > 0) {
#pragma unroll
      for (int i = 0; i < (int)(kUnit * sizeof(T) / 16); ++i)
        reinterpret_cast<u32x4*>(p)[i] = reinterpret_cast<const u32x4*>(t)[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kUnit; ++i)
      if (i < left) p[i] = t[i];
  }
}

// Sum over the lanes that share a row (a wave, or the workgroup through LDS).
template <int TPR, typename V>
__device__ __forceinline__ V row_sum(V v, V* red) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    v.x += __shfl_xor(v.x, d);
    v.y += __shfl_xor(v.y, d);
  }
  if constexpr (TPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    const V a = red[0], b = red[1], c = red[2], d = red[3];
    v.x = (a.x + b.x) + (c.x + d.x);
    v.y = (a.y + b.y) + (c.y + d.y);
  }
  return v;
}

__device__ __forceinline__ float sigmoid(float z) { return 1.0f / (1.0f + expf(-z)); }

// A row is shared by TPR lanes, UPT units each.
template <typename T, bool GATED, int TPR, int UPT>
__global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
  __shared__ float2 red[kThreads / 64];
  constexpr int kRows = kThreads / TPR;
  const int lane = threadIdx.x % TPR;
  Unit<T> kk[UPT], ww[UPT];
#pragma unroll
  for (int j = 0; j < UPT; ++j) {
    const int e = (lane + j * TPR) * kUnit, left = (int)a.width - e;
    kk[j].load((const T*)a.k + e, left, a.vec);
    ww[j].load((const T*)a.w + e, left, a.vec);
  }
  const uint64_t step = (uint64_t)gridDim.x * kRows;
  for (uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / TPR;; row += step) {
    // rows of one workgroup end together where they meet at a barrier
    if (row >= a.rows) break;
    Unit<T> ua[UPT], ub[UPT], uc[UPT];
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = (lane + j * TPR) * kUnit, left = (int)a.width - e;
      ua[j].load((const T*)a.a + row * a.a_row + e, left, a.vec);
      ub[j].load((const T*)a.b + row * a.b_row + e, left, a.vec);
      if constexpr (GATED) uc[j].load((const T*)a.c + row * a.c_row + e, left, a.vec);
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
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = (lane + j * TPR) * kUnit, left = (int)a.width - e;
      if constexpr (!GATED) store_unit((T*)a.r_new + row * a.width + e, v[j], left, a.vec);
      float u[kUnit];
#pragma unroll
      for (int i = 0; i < kUnit; ++i) u[i] = v[j][i] * k * ww[j].get(i);
      store_unit((T*)a.u + row * a.width + e, u, left, a.vec);
    }
  }
}

// Gradients.  The sums over rows (dk: skip or scale; dw) go to one fp32 row
// per workgroup, added up by k_norm_parts: no atomics, so a result does not
// depend on the order of execution.  A row's two sums and the difference
// g - v k^2 mean(g v) are fp64: where g is nearly parallel to v (always, in a
// row of one channel) the difference is far smaller than its terms.
template <typename T, bool GATED, int TPR, int UPT>
__global__ __launch_bounds__(kThreads) void k_norm_grad(NormArgs a) {
  __shared__ double2 red[kThreads / 64];
  __shared__ float part[TPR == 64 ? 2 * 64 * UPT * kUnit : 1];
  constexpr int kRows = kThreads / TPR;
  const int lane = threadIdx.x % TPR;
  Unit<T> kk[UPT], ww[UPT];
  float dk[UPT][kUnit], dw[UPT][kUnit];
#pragma unroll
  for (int j = 0; j < UPT; ++j) {
    const int e = (lane + j * TPR) * kUnit, left = (int)a.width - e;
    kk[j].load((const T*)a.k + e, left, a.vec);
    ww[j].load((const T*)a.w + e, left, a.vec);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) dk[j][i] = dw[j][i] = 0.0f;
  }
  const uint64_t step = (uint64_t)gridDim.x * kRows;
  for (uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < a.rows; row += step) {
    Unit<T> ua[UPT], ub[UPT], uc[UPT], ud[UPT], ur[UPT];
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = (lane + j * TPR) * kUnit, left = (int)a.width - e;
      ua[j].load((const T*)a.a + row * a.a_row + e, left, a.vec);
      ub[j].load((const T*)a.b + row * a.b_row + e, left, a.vec);
      if constexpr (GATED) uc[j].load((const T*)a.c + row * a.c_row + e, left, a.vec);
      ud[j].load((const T*)a.du + row * a.du_row + e, a.du ? left : 0, a.vec);
      if constexpr (!GATED)
        ur[j].load((const T*)a.dr_new + row * a.dr_row + e, a.dr_new ? left : 0, a.vec);
    }
    double2 sum = make_double2(0.0, 0.0);
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        float v;
        if constexpr (GATED) {
          const float z = uc[j].get(i);
          v = __builtin_fmaf(kk[j].get(i), ub[j].get(i), ua[j].get(i)) * (z * sigmoid(z));
        } else {
          v = __builtin_fmaf(kk[j].get(i), ua[j].get(i), ub[j].get(i));
        }
        sum.x = __builtin_fma((double)v, (double)v, sum.x);
        sum.y = __builtin_fma((double)(ud[j].get(i) * ww[j].get(i)), (double)v, sum.y);
      }
    }
    sum = row_sum<TPR>(sum, red);
    const double mean = sum.x / a.width + a.eps, c = sum.y / a.width / mean;
    const float k = 1.0f / sqrtf((float)mean);
#pragma unroll
    for (int j = 0; j < UPT; ++j) {
      const int e = (lane + j * TPR) * kUnit, left = (int)a.width - e;
      float o1[kUnit], o2[kUnit], o3[kUnit];
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        const float du = ud[j].get(i), kv = kk[j].get(i);
        if constexpr (GATED) {
          const float z = uc[j].get(i), sg = sigmoid(z), gate = z * sg, x = ub[j].get(i);
          const float q = __builtin_fmaf(kv, x, ua[j].get(i)), v = q * gate;
          const float dv = k * (float)__builtin_fma(-(double)v, c, (double)(du * ww[j].get(i)));
          const float dq = dv * gate;
          dw[j][i] = __builtin_fmaf(du, v * k, dw[j][i]);
          dk[j][i] = __builtin_fmaf(x, dq, dk[j][i]);
          o1[i] = dq;
          o2[i] = kv * dq;
          o3[i] = dv * q * __builtin_fmaf(gate, 1.0f - sg, sg);
        } else {
          const float o = ua[j].get(i);
          const float v = __builtin_fmaf(kv, o, ub[j].get(i));
          const float dp = (float)__builtin_fma(-(double)v, c, (double)(du * ww[j].get(i)));
          const float dv = __builtin_fmaf(k, dp, ur[j].get(i));
          dw[j][i] = __builtin_fmaf(du, v * k, dw[j][i]);
          dk[j][i] = __builtin_fmaf(o, dv, dk[j][i]);
          o1[i] = kv * dv;
          o2[i] = dv;
        }
      }
      store_unit((T*)a.da + row * a.width + e, o1, left, a.vec);
      store_unit((T*)a.db + row * a.width + e, o2, left, a.vec);
      if constexpr (GATED) store_unit((T*)a.dc + row * a.width + e, o3, left, a.vec);
    }
  }
  float* out = a.part + (uint64_t)blockIdx.x * 2 * a.width;
  if constexpr (TPR == 64) {
    constexpr int W = 64 * UPT * kUnit;
    for (int w = 0; w < kRows; ++w) {
      if ((int)(threadIdx.x / 64) == w) {
#pragma unroll
        for (int j = 0; j < UPT; ++j) {
#pragma unroll
          for (int i = 0; i < kUnit; ++i) {
            const int e = (lane + j * 64) * kUnit + i;
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
        const int e = (lane + j * TPR) * kUnit + i;
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
    for (uint32_t r = grp; r < a.blocks; r += 16) s += p[(uint64_t)r * 2 * a.width];
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

// A wave holds rows of up to 2048 channels (32 per lane), a workgroup longer ones.
template <typename T, bool GATED, bool GRAD>
hipError_t norm(const NormArgs& a, uint32_t blocks, hipStream_t s) {
  const uint32_t units = (a.width + kUnit - 1) / kUnit;
#define RUN(TPR, UPT)                                                       \
  do {                                                                      \
    if constexpr (GRAD)                                                     \
      k_norm_grad<T, GATED, TPR, UPT><<<blocks, kThreads, 0, s>>>(a);       \
    else                                                                    \
      k_norm<T, GATED, TPR, UPT><<<blocks, kThreads, 0, s>>>(a);            \
  } while (0)
  if (units <= 64) RUN(64, 1);
  else if (units <= 128) RUN(64, 2);
  else if (units <= 192) RUN(64, 3);
  else if (units <= 256) RUN(64, 4);
  else if (units <= 512) RUN(256, 2);
  else if (units <= 1024) RUN(256, 4);
  else RUN(256, 8);
#undef RUN
  return hipGetLastError();
}

uint32_t rows_per_block(uint32_t width) { return width <= 2048 ? 4 : 1; }

}  // namespace

uint32_t norm_grad_blocks(uint64_t rows, uint32_t width) {
  const uint64_t n = (rows + rows_per_block(width) - 1) / rows_per_block(width);
  return (uint32_t)(n < 512 ? n : 512);
}

hipError_t launch_norm(uint32_t dtype, bool gated, const NormArgs& a, hipStream_t s) {
  const uint64_t n = (a.rows + rows_per_block(a.width) - 1) / rows_per_block(a.width);
  const uint32_t blocks = (uint32_t)(n < 2048 ? n : 2048);
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
