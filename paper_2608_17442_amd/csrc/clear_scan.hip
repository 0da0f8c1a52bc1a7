// The gated linear recurrence in the clear and its gradient.
//
//   S_t = e^{la_t} S_{t-1} + x_t B_t^T,   y_t = S_t C_t        (per head, S in R^{P x N})
//
// is computed in chunks of kChunk tokens.  With cum_s the sum of la from the
// chunk's start up to and including s, and S the state that enters the chunk,
//
//   y_s = sum_{r <= s} e^{cum_s - cum_r} (C_s . B_r) x_r + e^{cum_s} S C_s
//   S'  = e^{cum_Q} S + sum_r e^{cum_Q - cum_r} x_r B_r^T
//
// so the work is matrix products over 64 x 64 x N tiles (MFMA), and the state
// stays in registers, in fp32, from chunk to chunk.  In bfloat16 the matrix instructions
// take eight bits of an operand.  Operands that are not inputs (the state, the weighted
// products C_s . B_r, the weighted inputs) enter as parts: two, within 2^-18 of the fp32
// value, so that an output is rounded once, when it is stored; the weighted inputs of a
// state (or of its gradient) that is an output of the call in three, which sum to the fp32
// value exactly.
#include <algorithm>
#include <type_traits>

#include "clear.hpp"
#include "clear_mem.hpp"
#include "fesc_internal.hpp"

namespace fesc {

namespace {

constexpr int Q = kChunk;
constexpr int PT = kPTile;

// A matrix operand as the 16x16 tiles take it: lane l holds row (or column)
// l % 16 and 8 of the 32 values along the axis that is summed over, which 8
// being the same for both operands of a product.
template <typename T>
struct Elem;
template <>
struct Elem<__bf16> {
  using Frag = bf16x8;
  using Four = bf16x4;
  static constexpr int kUnit = 8;  // elements in 16 bytes
  // Row padding of LDS tiles.  A row pitch of 8 words past a multiple of 32
  // words puts the 8 rows of a 16-byte access, and the 4 rows of a
  // transposing access, on distinct banks.
  static constexpr int kPad = 16;
};
template <>
struct Elem<float> {
  using Frag = f32x8;
  using Four = f32x4;
  static constexpr int kUnit = 4;
  static constexpr int kPad = 4;
};

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const f32x8& a, const f32x8& b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// Eight values that lie next to each other in an LDS row.
__device__ __forceinline__ bf16x8 row_frag(const __bf16* p) {
  return *reinterpret_cast<const bf16x8*>(p);
}
__device__ __forceinline__ f32x8 row_frag(const float* p) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p);
  const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
  return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// Four values of one column of an LDS tile: rows row0 .. row0 + 3 at column
// col0 + l % 16, row0 the same for the 16 lanes of a group.
__device__ __forceinline__ bf16x4 col_four(const __bf16* tile, int pitch, int row0, int col0) {
  const int i = threadIdx.x & 15;
  const __bf16* p = tile + (row0 + (i >> 2)) * pitch + col0 + 4 * (i & 3);
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(p));
  return __builtin_bit_cast(bf16x4, v);
}
__device__ __forceinline__ f32x4 col_four(const float* tile, int pitch, int row0, int col0) {
  const float* p = tile + row0 * pitch + col0 + (threadIdx.x & 15);
  return f32x4{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
}

// The same for the columns of state tile t: lane 4 j + i of a group takes column
// state_col(t, j) + i.
__device__ __forceinline__ constexpr int state_col(int t, int j) {
  return 32 * (t / 2) + 8 * j + 4 * (t & 1);
}
__device__ __forceinline__ bf16x4 state_four(const __bf16* tile, int pitch, int row0, int t) {
  const int i = threadIdx.x & 15;
  const __bf16* p = tile + (row0 + (i >> 2)) * pitch + state_col(t, i & 3);
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(p));
  return __builtin_bit_cast(bf16x4, v);
}
__device__ __forceinline__ f32x4 state_four(const float* tile, int pitch, int row0, int t) {
  const int i = threadIdx.x & 15;
  const float* p = tile + row0 * pitch + state_col(t, i >> 2) + (i & 3);
  return f32x4{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
}

__device__ __forceinline__ bf16x8 join(const bf16x4& a, const bf16x4& b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x8 join(const f32x4& a, const f32x4& b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The parts of a fp32 operand in the call's type: itself, or COUNT bf16 values.
// Three, each the leading 8 bits of what the ones before leave, sum to it
// exactly; two, each rounded to nearest, to within 2^-18 of it.
template <typename T, int COUNT>
struct Parts;
template <int COUNT>
struct Parts<float, COUNT> {
  static constexpr int kCount = 1;
  f32x8 p[1];
  __device__ __forceinline__ void split(const f32x4& a, const f32x4& b) { p[0] = join(a, b); }
};
template <int COUNT>
struct Parts<__bf16, COUNT> {
  static constexpr int kCount = COUNT;
  bf16x8 p[COUNT];
  __device__ __forceinline__ void split(const f32x4& a, const f32x4& b) {
    f32x8 v = join(a, b);
    if constexpr (COUNT == 2) {
      p[0] = __builtin_convertvector(v, bf16x8);
      p[1] = __builtin_convertvector(v - __builtin_convertvector(p[0], f32x8), bf16x8);
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = __builtin_amdgcn_perm(__float_as_uint(v[2 * j + 1]), __float_as_uint(v[2 * j]),
                                       0x07060302u);
        p[k] = __builtin_bit_cast(bf16x8, w);
        if (k < 2) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            v[j] -= __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u);
        }
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  return (float)*p;
}

// Where a thread's units of a ROWS x COLS tile lie in memory: unit k in row `row` +
// k `rows_apart`; none of the thread's units where its column is absent.
// FIRST: the first thread of those that share the work.
template <typename T, int COLS, int THREADS, int FIRST = 0>
struct Rows {
  static constexpr int rows_apart = THREADS / (COLS / Elem<T>::kUnit);
  uint32_t pitch, first, step;
  int cols, row;
  __device__ __forceinline__ Rows(uint32_t pitch_, int cols_) : pitch(pitch_), cols(cols_) {
    constexpr int kUnit = Elem<T>::kUnit, kPerRow = COLS / kUnit;
    const int col = (threadIdx.x - FIRST) % kPerRow * kUnit;
    row = (threadIdx.x - FIRST) / kPerRow;
    first = (row * pitch + col) * (uint32_t)sizeof(T);
    step = rows_apart * pitch * (uint32_t)sizeof(T);
    if (col >= cols) row = 1 << 30;
  }
  // offset of whole unit k of `rows` rows
  __device__ __forceinline__ uint32_t at(int k, int rows) const {
    return row < rows - k * rows_apart ? first + k * step : kAbsent;
  }
};

// One unit of 16 bytes, as loaded.  Rows at any alignment: the 16 bytes from the
// word on in which the unit begins and the word behind them, or, of a row's last
// unit, of its last 16 bytes, so that every word read holds an element of the row;
// `by`: how many elements it lies too far up.
template <bool VEC>
struct Loaded {
  u32x4 w;
};
template <>
struct Loaded<false> {
  u32x4 w;
  uint32_t more, by;
};
template <typename T>
__device__ __forceinline__ u32x4 settled(const Loaded<true>& l) {
  return l.w;
}
template <typename T>
__device__ __forceinline__ u32x4 settled(const Loaded<false>& l) {
  uint32_t v[8] = {l.w[0], l.w[1], l.w[2], l.w[3], 0, 0, 0, 0};
  if constexpr (sizeof(T) == 2) v[4] = l.more & 0xffffu;
  const uint32_t words = sizeof(T) == 2 ? l.by >> 1 : l.by;
#pragma unroll
  for (int d = 4; d >= 1; d /= 2) {
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = words & d ? (i + d < 5 ? v[i + d] : 0) : v[i];
  }
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = sizeof(T) == 2 ? __builtin_amdgcn_alignbyte(v[i + 1], v[i], (l.by & 1) * 2) : v[i];
  return o;
}

// Registers of one thread for a tile of ROWS x COLS elements on its way from
// global memory to LDS; rows and columns past the valid ones are zero.
template <typename T, int ROWS, int COLS, int THREADS, bool VEC, int FIRST = 0>
struct Stage {
  static constexpr int kUnit = Elem<T>::kUnit;
  static constexpr int kPerRow = COLS / kUnit;
  static constexpr int kUnits = ROWS * kPerRow / THREADS;
  static_assert(ROWS * kPerRow % THREADS == 0, "whole units per thread");
  using In = Rows<T, COLS, THREADS, FIRST>;
  Loaded<VEC> r[kUnits];

  __device__ __forceinline__ void load(const T* base, const In& in, int rows) {
    if constexpr (VEC) {
      const Mem m(base);
#pragma unroll
      for (int k = 0; k < kUnits; ++k) r[k].w = m.load16(in.at(k, rows));
    } else if (in.cols < kUnit) {  // rows of a few elements: one at a time
      const Mem m(base);
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const int i = (threadIdx.x - FIRST) + k * THREADS;
        const int row = i / kPerRow, col = i % kPerRow * kUnit;
        const uint32_t at = (row * in.pitch + col) * (uint32_t)sizeof(T);
        u32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
          const uint32_t w = m.load_bits<T>(
              row < rows && col + j < in.cols ? at + j * (uint32_t)sizeof(T) : kAbsent);
          if constexpr (sizeof(T) == 4)
            v[j] = w;
          else
            v[j / 2] |= w << (16 * (j & 1));
        }
        r[k] = {v, 0, 0};
      }
    } else {
      const uint32_t off = reinterpret_cast<uintptr_t>(base) & 3;
      const Mem m(reinterpret_cast<const char*>(base) - off);
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const int i = (threadIdx.x - FIRST) + k * THREADS;
        const int row = i / kPerRow, col = i % kPerRow * kUnit;
        const int from = min(col, in.cols - kUnit);
        const uint32_t at = off + (row * in.pitch + from) * (uint32_t)sizeof(T);
        const bool seen = row < rows && col < in.cols;
        const uint32_t odd = sizeof(T) == 2 ? at >> 1 & 1 : 0;
        r[k].w = m.load16(seen ? at & ~3u : kAbsent);
        r[k].more = sizeof(T) == 2 ? m.load_bits<float>(seen && odd ? (at & ~3u) + 16 : kAbsent) : 0;
        r[k].by = col - from + odd;
      }
    }
  }
  __device__ __forceinline__ void store(T* tile, int pitch) const {
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int i = (threadIdx.x - FIRST) + k * THREADS;
      *reinterpret_cast<u32x4*>(tile + i / kPerRow * pitch + i % kPerRow * kUnit) = settled<T>(r[k]);
    }
  }
  __device__ __forceinline__ void take(const T* tile, int pitch) {
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int i = (threadIdx.x - FIRST) + k * THREADS;
      r[k].w = *reinterpret_cast<const u32x4*>(tile + i / kPerRow * pitch + i % kPerRow * kUnit);
    }
  }
  __device__ __forceinline__ void put(T* base, const In& out, int rows) const {
    if constexpr (VEC) {
      const Mem m(base);
#pragma unroll
      for (int k = 0; k < kUnits; ++k) m.store16(out.at(k, rows), r[k].w);
    } else {  // whole units word by word, at any alignment of elements
      const uint32_t off = reinterpret_cast<uintptr_t>(base) & 3;
      const Mem m(reinterpret_cast<char*>(base) - off);
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const int i = (threadIdx.x - FIRST) + k * THREADS;
        const int row = i / kPerRow, col = i % kPerRow * kUnit;
        const int left = row < rows ? out.cols - col : 0;
        const uint32_t at = off + (row * out.pitch + col) * (uint32_t)sizeof(T);
        const u32x4 v = r[k].w;
        const bool odd = sizeof(T) == 2 && (at & 2);
        m.store16(left >= kUnit && !odd ? at : kAbsent, v);
        if (left < kUnit || odd) {
#pragma unroll
          for (int j = 0; j < kUnit; ++j)
            m.store_bits<T>(j < left ? at + j * (uint32_t)sizeof(T) : kAbsent,
                            sizeof(T) == 4 ? v[j * sizeof(T) / 4]
                                           : v[j * sizeof(T) / 4] >> (16 * (j & 1)) & 0xffffu);
        }
      }
    }
  }
};

// Running sums of the log decays (base 2) of a chunk, lane l the token l, in
// fp64 and then as a pair of floats: hi a multiple of 2^-6, so that hi_s - hi_r
// is exact and a difference of two sums is as accurate as a sum over the
// tokens between them, whatever lies before them.  la below kReset (in
// particular -inf: a reset) counts as kReset, whose decay is 0 in fp32.
constexpr float kReset = -1000.0f;
struct Cum {
  float hi, lo;   // of token l
  float e, w;     // e^{cum_l}, e^{cum_Q - cum_l}
  float total;    // e^{cum_Q}
};
__device__ __forceinline__ float exp2_diff(float hs, float ls, float hr, float lr) {
  return __builtin_amdgcn_exp2f((hs - hr) + (ls - lr));
}
// The same where `seen`, else 0 (without a branch around the exponential).
__device__ __forceinline__ float exp2_seen(bool seen, float hs, float ls, float hr, float lr) {
  const float d = (hs - hr) + (ls - lr);
  return __builtin_amdgcn_exp2f(seen ? d : -INFINITY);
}
// v decayed; a decay of 0 forgets v whatever it is, not finite included.
__device__ __forceinline__ float decayed(float decay, float v) {
  return decay == 0.0f ? 0.0f : decay * v;
}
__device__ __forceinline__ f32x4 decayed(float decay, const f32x4& v) {
  f32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = decayed(decay, v[i]);
  return o;
}
// The wave's number, known to be the same for all its lanes.
__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}
// One step of the scan over a wave: adds the value that the DPP control moves
// here (0 where it moves none).
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double c) {
  const uint64_t w = __builtin_bit_cast(uint64_t, c);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)w, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(w >> 32), CTRL, ROWS, 0xf, false);
  return c + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ Cum cumulate(float la) {
  constexpr double kLog2e = 1.4426950408889634;
  double c = (double)(la < kReset ? kReset : la) * kLog2e;
  c = dpp_add<0x111, 0xf>(c);  // row_shr 1, 2, 4, 8: sums within 16 lanes
  c = dpp_add<0x112, 0xf>(c);
  c = dpp_add<0x114, 0xf>(c);
  c = dpp_add<0x118, 0xf>(c);
  c = dpp_add<0x142, 0xa>(c);  // row_bcast 15 to rows 1 and 3
  c = dpp_add<0x143, 0xc>(c);  // row_bcast 31 to rows 2 and 3
  Cum r;
  r.hi = (float)(__builtin_rint(c * 64.0) * (1.0 / 64.0));
  r.lo = (float)(c - (double)r.hi);
  const float th = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__float_as_uint(r.hi), 63));
  const float tl = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__float_as_uint(r.lo), 63));
  r.e = exp2_diff(r.hi, r.lo, 0.0f, 0.0f);
  r.w = exp2_diff(th, tl, r.hi, r.lo);
  r.total = __builtin_amdgcn_exp2f(th + tl);
  return r;
}

// ------------------------------------------------------------ scan kernels

// One workgroup: HB neighbouring channel tiles (heads, where a head has one
// tile) of one group over the chunks of one segment; what it reads of B and C
// serves all of them.  Of each, wave 4 e + w (e < EW) holds the state rows
// p = 16 w + l % 16, of them part e of the entries n, as transposed MFMA result
// tiles t = e kOwn ... (e + 1) kOwn - 1 with n = state_col(t, g) + i (g = l / 16):
// tiles 2 q and 2 q + 1 together are, in registers, the operand
// S[p][32 q + 8 g ...] of the product with C.
// The registers are held to two workgroups on a compute unit: in bfloat16, as LDS
// has no room for a second one in float32, and of the output kernel on aligned rows,
// as others take more.
template <typename T, int NT, int HB, int EW>
struct ScanTiles {
  static constexpr int XS = PT + Elem<T>::kPad;
  static constexpr int NS = NT + Elem<T>::kPad;
  static constexpr int kThreads = 256 * EW;
  static constexpr int kOwn = NT / 16 / EW;  // state tiles of a wave, per channel tile
};

// Workgroups that read the same B and C rows lie `batch * segs` apart: on one
// XCD where that is a multiple of 8.
struct Where {
  uint32_t b, v, seg, g;  // v: first channel tile, among those of all heads
  template <int HB>
  __device__ __forceinline__ static Where of(const ScanShape& sh) {
    Where w;
    const uint32_t per = sh.batch * sh.segs, bs = blockIdx.x % per;
    w.b = bs / sh.segs;
    w.seg = bs % sh.segs;
    w.v = blockIdx.x / per * HB;
    w.g = w.v / sh.ptiles / (sh.heads / sh.groups);
    return w;
  }
};
// The channel tile whose running sums a wave forms, -1: none.  Of the output
// kernel's waves these have least to do with G.
template <int HB, int EW>
__device__ __forceinline__ int sums_tile() {
  const int h = wave_id() - 4 * (EW - 1);
  return h >= 0 && h < HB ? h : -1;
}

// One channel tile of a workgroup.
struct Head {
  uint32_t h;     // head
  int p0, rows;   // first channel, channels
  uint64_t at;    // batch * heads + head
  __device__ __forceinline__ Head(const ScanShape& sh, const Where& w, int k) {
    const uint32_t v = w.v + k;
    h = v / sh.ptiles;
    p0 = v % sh.ptiles * PT;
    rows = min(PT, (int)sh.head_dim - p0);
    at = (uint64_t)w.b * sh.heads + h;
  }
};

// A wave's part of a state, tiles t0 ..., from and to memory.
template <bool VEC, int NTILES>
__device__ __forceinline__ void load_state(f32x4 (&s)[NTILES], const float* base, int p, int rows,
                                           int N, int t0) {
  const int g = (threadIdx.x & 63) >> 4;
  const Mem m(base);
#pragma unroll
  for (int t = 0; t < NTILES; ++t) {
    const int n = state_col(t0 + t, g);
    s[t] = m.load_four<VEC>((p * N + n) * 4, p < rows ? N - n : 0);
  }
}
// The state that enters segment `seg` of a head.  Joined: as k_scan_join left it.
// Otherwise from the summaries of the segments before, the summary of segment j
// lying in the place of segment j + 1.
template <bool VEC, int NTILES>
__device__ __forceinline__ void enter_segment(f32x4 (&s)[NTILES], const ScanShape& sh,
                                              const ScanDir& d, uint64_t head, uint32_t seg,
                                              int p0, int p, int rows, int t0) {
  const int N = sh.d_state;
  const uint64_t size = (uint64_t)sh.head_dim * N, tile = (uint64_t)p0 * N;
  const float* from = d.init ? d.init + head * size : nullptr;
  const float* segs = d.seg_states ? d.seg_states + head * sh.segs * size : nullptr;
  if (sh.joined && segs) from = segs + seg * size;
  if (from) {
    load_state<VEC>(s, from + tile, p, rows, N, t0);
  } else {
#pragma unroll
    for (int t = 0; t < NTILES; ++t) s[t] = f32x4{0, 0, 0, 0};
  }
  if (sh.joined || !segs) return;
  constexpr int kAtOnce = NTILES <= 4 ? 4 : 2;  // loads under way
  for (uint32_t j0 = 1; j0 <= seg; j0 += kAtOnce) {
    f32x4 own[kAtOnce][NTILES];
    float decay[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {  // past the last: nothing, kept as it is
      const uint32_t j = min(j0 + k, seg);
      load_state<VEC>(own[k], segs + j * size + tile, p, j0 + k <= seg ? rows : 0, N, t0);
      decay[k] = j0 + k <= seg ? d.seg_decay[head * sh.segs + j - 1] : 1.0f;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
#pragma unroll
      for (int t = 0; t < NTILES; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][i] = __builtin_fmaf(decay[k], decay[k] == 0.0f ? 0.0f : s[t][i], own[k][t][i]);
      }
    }
  }
}
template <bool VEC, int NTILES>
__device__ __forceinline__ void store_state(const f32x4 (&s)[NTILES], float* base, int p, int rows,
                                            int N, int t0) {
  const int g = (threadIdx.x & 63) >> 4;
  const Mem m(base);
#pragma unroll
  for (int t = 0; t < NTILES; ++t) {
    const int n = state_col(t0 + t, g);
    m.store_four<float, VEC>((p * N + n) * 4u, s[t], p < rows ? N - n : 0);
  }
}

// Where the chunk states that a gradient reads keep what lane `lane` holds of tile t of
// the rows 16 w ...: bytes from the channel tile's first one, whole lines per access.
__device__ __forceinline__ uint32_t kept_at(int w, int t, int lane, int entries) {
  return ((w * (entries / 16) + t) * 64 + lane) * 16;
}

// The operand with the tokens of half q of a chunk along the summed axis, from
// a tile's columns col0 ...: tokens 32 q + 4 g + i and 32 q + 16 + 4 g + i.
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag token_frag(const T* tile, int pitch, int q,
                                                             int col0) {
  const int r = 32 * q + 4 * ((threadIdx.x & 63) >> 4);
  return join(col_four(tile, pitch, r, col0), col_four(tile, pitch, r + 16, col0));
}
__device__ __forceinline__ f32x4 half(const bf16x8& v, int k) {
  return k ? f32x4{(float)v[4], (float)v[5], (float)v[6], (float)v[7]}
           : f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}
__device__ __forceinline__ f32x4 half(const f32x8& v, int k) {
  return k ? f32x4{v[4], v[5], v[6], v[7]} : f32x4{v[0], v[1], v[2], v[3]};
}

// S' = total S + sum_r w_r x_r B_r^T over the chunk in LDS; xf: this wave's rows
// of x as operands.  Two state tiles at a time, whose products do not wait for
// each other's sums.
template <typename T, int NT, int PARTS, int HB, int OWN>
__device__ __forceinline__ void update_state(f32x4 (&s)[HB][OWN],
                                             const typename Elem<T>::Frag (&xf)[HB][2],
                                             const T* bs, const float (&w)[HB][Q],
                                             const float (&total)[HB], int t0) {
  constexpr int NS = NT + Elem<T>::kPad;
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    const float e = total[h];
#pragma unroll
    for (int t = 0; t < OWN; ++t) s[h][t] = decayed(e, s[h][t]);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int r = 32 * q + 4 * g;
    Parts<T, PARTS> x[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h)
      x[h].split(half(xf[h][q], 0) * *reinterpret_cast<const f32x4*>(w[h] + r),
                 half(xf[h][q], 1) * *reinterpret_cast<const f32x4*>(w[h] + r + 16));
#pragma unroll
    for (int t = 0; t < OWN; t += 2) {
      typename Elem<T>::Frag b[2];
#pragma unroll
      for (int f = 0; f < 2; ++f)
        b[f] = join(state_four(bs, NS, r, t0 + t + f), state_four(bs, NS, r + 16, t0 + t + f));
#pragma unroll
      for (int k = 0; k < Parts<T, PARTS>::kCount; ++k) {
#pragma unroll
        for (int h = 0; h < HB; ++h) {
#pragma unroll
          for (int f = 0; f < 2; ++f) s[h][t + f] = mma(b[f], x[h].p[k], s[h][t + f]);
        }
      }
    }
  }
}

// States only.  Segment pass (`summaries`): each segment's own state, from
// zero, and its total decay, to seg_states and seg_decay.  Otherwise from the
// state that enters the segment: the states that enter the chunks, and the
// final state.  Chunks lie in LDS in turn in two places: one barrier each.
// blockIdx.y: the NT entries of the state at hand.
template <typename T, int NT, bool VEC, int PARTS, int HB, int EW>
__global__ __launch_bounds__(256 * EW, HB * EW == 1 ? 3 : (sizeof(T) == 2 ? 2 : 1) * EW)
    void k_scan_states(ScanShape sh, ScanDir d0, ScanDir d1, bool summaries) {
  using Tiles = ScanTiles<T, NT, HB, EW>;
  constexpr int kThreads = Tiles::kThreads;
  constexpr int XS = Tiles::XS, NS = Tiles::NS;
  __shared__ __align__(16) T xs[2][HB][Q * XS];
  __shared__ __align__(16) T bs[2][Q * NS];
  __shared__ __align__(16) float wt[2][HB][Q];
  __shared__ float total[2][HB];
  const ScanDir& d = blockIdx.z ? d1 : d0;
  const Where at = Where::of<HB>(sh);
  const int wave = wave_id() & 3, part = wave_id() >> 2, t0 = part * Tiles::kOwn;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int sums_of = sums_tile<HB, EW>();  // whose running sums this wave forms
  const int P = sh.head_dim, N = sh.d_state, p = 16 * wave + (lane & 15);
  const int n0 = blockIdx.y * NT, m0 = t0 + n0 / 16;  // first entry and tile in the state
  // segments and chunks are counted in the direction of the pass
  const int first = at.seg * sh.seg_chunks;
  const int count = min((int)sh.seg_chunks, (int)sh.chunks - first);
  if (summaries && at.seg + 1 == sh.segs) return;  // no segment follows the last
  const uint64_t size = (uint64_t)P * N;
  const T* u = (const T*)d.u + at.b * d.u_batch;
  const T* v = (const T*)d.v + at.b * d.v_batch + (int64_t)at.g * N + n0;
  const T* la = (const T*)sh.la + at.b * sh.la_batch + Head(sh, at, sums_of < 0 ? 0 : sums_of).h;

  f32x4 s[HB][Tiles::kOwn];
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    const Head hd(sh, at, h);
    if (summaries) {
#pragma unroll
      for (int t = 0; t < Tiles::kOwn; ++t) s[h][t] = f32x4{0, 0, 0, 0};
    } else {
      enter_segment<VEC>(s[h], sh, d, hd.at, at.seg, hd.p0, p, hd.rows, m0);
    }
  }
  using XStage = Stage<T, Q, PT, kThreads, VEC>;
  using NStage = Stage<T, Q, NT, kThreads, VEC>;
  XStage xst[HB];
  NStage bst;
  const typename NStage::In bin(d.v_token, min(NT, N - n0));
  float lav = 0.0f;  // log decay of token `lane` of that tile
  const uint32_t la_at = lane * (uint32_t)sh.la_token * (uint32_t)sizeof(T);
  auto chunk = [&](int k) { return d.reverse ? (int)sh.chunks - 1 - (first + k) : first + k; };
  auto fetch = [&](int k) {
    const int64_t start = (int64_t)chunk(k) * Q;
    const int n = min((int64_t)Q, (int64_t)sh.len - start);
    if (sums_of >= 0)
      lav = Mem(la + start * sh.la_token).load<T>(lane < n ? la_at : kAbsent);
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      const Head hd(sh, at, h);
      xst[h].load(u + start * d.u_token + (int64_t)hd.h * P + hd.p0,
                  typename XStage::In(d.u_token, hd.rows), n);
    }
    bst.load(v + start * d.v_token, bin, n);
  };
  auto place = [&](int k) {
    if (sums_of >= 0) {
      const Cum cum = cumulate(lav);
      wt[k & 1][sums_of][lane] = d.reverse ? cum.e : cum.w;
      if (lane == 0) total[k & 1][sums_of] = cum.total;
    }
#pragma unroll
    for (int h = 0; h < HB; ++h) xst[h].store(xs[k & 1][h], XS);
    bst.store(bs[k & 1], NS);
    __syncthreads();
  };
  fetch(0);
  place(0);
  float decay[HB];
#pragma unroll
  for (int h = 0; h < HB; ++h) decay[h] = 1.0f;
  for (int k = 0; k < count; ++k) {
    if (k + 1 < count) fetch(k + 1);
    if (d.chunk_states && !summaries) {
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        const Head hd(sh, at, h);
        const Mem m(d.chunk_states + sh.chunk_state(hd.at, chunk(k), hd.p0 / PT));
#pragma unroll
        for (int t = 0; t < Tiles::kOwn; ++t)
          m.store16(p < hd.rows && state_col(m0 + t, g) < N
                        ? kept_at(wave, m0 + t, lane, sh.kept_entries()) : kAbsent,
                    __builtin_bit_cast(u32x4, s[h][t]));
      }
    }
    typename Elem<T>::Frag xf[HB][2];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
#pragma unroll
      for (int q = 0; q < 2; ++q) xf[h][q] = token_frag(xs[k & 1][h], XS, q, 16 * wave);
      decay[h] *= total[k & 1][h];
    }
    update_state<T, NT, PARTS, HB>(s, xf, bs[k & 1], wt[k & 1], total[k & 1], t0);
    if (k + 1 < count) place(k + 1);
  }
#pragma unroll
  for (int h = 0; h < HB; ++h) {
    const Head hd(sh, at, h);
    const uint64_t tile = (uint64_t)hd.p0 * N;
    if (summaries) {
      store_state<VEC>(s[h], d.seg_states + (hd.at * sh.segs + at.seg + 1) * size + tile, p,
                       hd.rows, N, m0);
      if (threadIdx.x == 0 && hd.p0 == 0 && n0 == 0)
        d.seg_decay[hd.at * sh.segs + at.seg] = decay[h];
    } else if (d.fin && at.seg + 1 == sh.segs) {
      store_state<VEC>(s[h], d.fin + hd.at * size + tile, p, hd.rows, N, m0);
    }
  }
}

// Segment summaries to the states that enter the segments, in place: the
// summary of segment j lies in the place of segment j + 1.  Bound by memory: 66 MB
// (24 heads, 42 segments) in 12 us.
__global__ __launch_bounds__(256) void k_scan_join(ScanShape sh, ScanDir d0, ScanDir d1) {
  const ScanDir& d = blockIdx.z ? d1 : d0;
  const uint32_t size = sh.head_dim * sh.d_state, blocks = (size + 255) / 256;
  const uint32_t e = blockIdx.x % blocks * 256 + threadIdx.x;
  const uint64_t head = blockIdx.x / blocks;
  if (e >= size) return;
  float* s = d.seg_states + head * sh.segs * (uint64_t)size + e;
  const float* decay = d.seg_decay + head * sh.segs;
  float carry = d.init ? d.init[head * size + e] : 0.0f;
  s[0] = carry;
  constexpr uint32_t kAtOnce = 8;  // loads under way
  for (uint32_t j0 = 1; j0 < sh.segs; j0 += kAtOnce) {
    float own[kAtOnce], keep[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t j = min(j0 + k, sh.segs - 1);
      own[k] = s[(uint64_t)j * size];
      keep[k] = decay[j - 1];
    }
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      carry = __builtin_fmaf(keep[k], keep[k] == 0.0f ? 0.0f : carry, own[k]);
      if (j0 + k < sh.segs) s[(uint64_t)(j0 + k) * size] = carry;
    }
  }
}

// Outputs and final state.  Per chunk: wave 4 e + w forms, for the tokens of tile w,
// the columns of G^T, G = C B^T, of the tokens r of half e, and writes their products
// with the decays to LDS; meanwhile, from its part of the state, a part of y^T for its 16
// channels and all tokens, of which it hands the tokens of half 1 - e to the other
// wave with these channels; and its part of the new state.  Then, for the tokens of half e,
// the chunk's own part of y^T from what all waves wrote.
// Bound by the way from barrier to barrier, on which LDS, the matrix pipe and the
// issue of instructions take turns: 8 x 2048 tokens, 24 heads of 64, state 128, 88 us
// (25 at a copy's rate); 50001 tokens in 42 segments 76 + 13 + 205 us (68).  Operands in one
// part and rounded: 75 and 195 us in all.
template <typename T, int NT, bool VEC, int PARTS>
__global__ __launch_bounds__(512, sizeof(T) == 2 && VEC ? 4 : 2) void k_scan_out(ScanShape sh,
                                                                                 ScanDir d,
                                                                                 ScanOut o) {
  constexpr int EW = 2;
  using Tiles = ScanTiles<T, NT, 1, EW>;
  constexpr int kThreads = Tiles::kThreads, kOwn = Tiles::kOwn;
  constexpr int XS = Tiles::XS, NS = Tiles::NS;
  constexpr int NQ = NT / 32;
  using Frag = typename Elem<T>::Frag;
  using Two = Parts<T, 2>;
  constexpr int kParts = Two::kCount;
  // The weighted products: rows s of 32 or, in the second half, 64 tokens r.
  constexpr int kRow = 16 / sizeof(T), LS0 = 32 + kRow, LS1 = 64 + kRow, kLg = 32 * (LS0 + LS1);
  __shared__ __align__(16) T xs[Q * XS];
  __shared__ __align__(16) T bs[Q * NS];
  __shared__ __align__(16) T cs[Q * NS];
  __shared__ __align__(16) T lg[kParts][kLg];
  __shared__ __align__(16) f32x4 ex[2][8][64];  // what is handed over, by lanes
  __shared__ __align__(16) float hi[2][Q], lo[2][Q], wt[2][1][Q];
  __shared__ float total[2][1];
  const Where where = Where::of<1>(sh);
  const Head at(sh, where, 0);
  const int wave = wave_id() & 3, part = wave_id() >> 2, t0 = part * kOwn;
  const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  const bool sums_here = wave_id() == 4;  // of the waves with least to do with G
  const int P = sh.head_dim, N = sh.d_state, p = 16 * wave + col;
  const int first = where.seg * sh.seg_chunks;
  const int count = min((int)sh.seg_chunks, (int)sh.chunks - first);
  const uint64_t size = (uint64_t)P * N;
  const T* u = (const T*)d.u + where.b * d.u_batch + (int64_t)at.h * P + at.p0;
  const T* v = (const T*)d.v + where.b * d.v_batch + (int64_t)where.g * N;
  const T* cc = (const T*)o.c + where.b * o.c_batch + (int64_t)where.g * N;
  const T* la = (const T*)sh.la + where.b * sh.la_batch + at.h;

  f32x4 s[1][kOwn];
  enter_segment<VEC>(s[0], sh, d, at.at, where.seg, at.p0, p, at.rows, t0);
  using XStage = Stage<T, Q, PT, kThreads, VEC>;
  using NStage = Stage<T, Q, NT, kThreads, VEC>;
  XStage xst;
  NStage bst, cst;
  const typename XStage::In xin(d.u_token, at.rows), yin(sh.heads * P, at.rows);
  const typename NStage::In bin(d.v_token, N), cin(o.c_token, N);
  auto start = [&](int k) { return (int64_t)(first + k) * Q; };
  auto tokens = [&](int k) { return (int)min((int64_t)Q, (int64_t)sh.len - start(k)); };
  // the next chunk's loads, in portions that do not hold the work up
  auto fetch_b = [&](int k) {
    if (k < count) bst.load(v + start(k) * d.v_token, bin, tokens(k));
  };
  auto fetch_c = [&](int k) {
    if (k < count) cst.load(cc + start(k) * o.c_token, cin, tokens(k));
  };
  auto fetch_x = [&](int k) {
    if (k < count) xst.load(u + start(k) * d.u_token, xin, tokens(k));
  };
  // Log decays come two chunks ahead from memory, their running sums one ahead
  // into LDS.
  uint32_t lav = 0;  // as loaded: a conversion would wait for it
  const uint32_t la_at = lane * (uint32_t)sh.la_token * (uint32_t)sizeof(T);
  auto fetch_la = [&](int k) {
    if (k < count)
      lav = Mem(la + start(k) * sh.la_token).load_bits<T>(lane < tokens(k) ? la_at : kAbsent);
  };
  auto sums = [&](int k) {
    const Cum cum = cumulate(Mem::value<T>(lav));
    hi[k & 1][lane] = cum.hi;
    lo[k & 1][lane] = cum.lo;
    wt[k & 1][0][lane] = cum.w;
    if (lane == 0) total[k & 1][0] = cum.total;
  };
  // outputs of a chunk, which lay in LDS in the place of its x, to memory
  auto put_y = [&](const XStage& y, int k) {
    y.put((T*)o.y + (((uint64_t)where.b * sh.len + start(k)) * sh.heads + at.h) * P + at.p0, yin,
          tokens(k));
  };
  if (sums_here) fetch_la(0);
  fetch_b(0);
  fetch_c(0);
  fetch_x(0);
  if (sums_here) {
    sums(0);
    fetch_la(1);
  }
  for (int k = 0; k < count; ++k) {
    const int now = k & 1;
    XStage y_out;
    if (k) {
      __syncthreads();
      y_out.take(xs, XS);
    }
    // a thread stores its x where it has read outputs
    xst.store(xs, XS);
    bst.store(bs, NS);
    cst.store(cs, NS);
    if (k) put_y(y_out, k - 1);  // behind the wait for the loads, which it need not wait for
    __syncthreads();
    if (sums_here && k + 1 < count) {
      sums(k + 1);
      fetch_la(k + 2);
    }
    fetch_b(k + 1);
    if (2 * part <= wave) {
      // rows r = 32 part + 16 f + 4 g + i, column s = 16 wave + col
      f32x4 w[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const Frag cf = row_frag(cs + (16 * wave + col) * NS + 32 * q + 8 * g);
#pragma unroll
        for (int f = 0; f < 2; ++f)
          w[f] = mma(row_frag(bs + (32 * part + 16 * f + col) * NS + 32 * q + 8 * g), cf, w[f]);
      }
      const float hs = hi[now][16 * wave + col], ls = lo[now][16 * wave + col];
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int r = 32 * part + 16 * f + 4 * g;
        const f32x4 hr = *reinterpret_cast<const f32x4*>(hi[now] + r);
        const f32x4 lr = *reinterpret_cast<const f32x4*>(lo[now] + r);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[f][i] *= exp2_seen(r + i <= 16 * wave + col, hs, ls, hr[i], lr[i]);
      }
      // position 32 e + 8 g + 4 f + i holds token 32 e + 16 f + 4 g + i, so that a row
      // read gives the operand that matches token_frag
      Two lw;
      lw.split(w[0], w[1]);
      const int at_s = wave < 2 ? (16 * wave + col) * LS0
                                : 32 * LS0 + (16 * wave + col - 32) * LS1 + 32 * part;
#pragma unroll
      for (int a = 0; a < kParts; ++a)
        *reinterpret_cast<Frag*>(lg[a] + at_s + 8 * g) = lw.p[a];
    }
    Frag xf[1][2];
#pragma unroll
    for (int q = 0; q < 2; ++q) xf[0][q] = token_frag(xs, XS, q, 16 * wave);
    // y^T: rows p = 16 wave + 4 g + i, columns s = 16 j + col; j: first the tokens that
    // are handed over, then this wave's own
    f32x4 in[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) in[j] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < kOwn; t += 2) {
      Two sf;
      sf.split(s[0][t], s[0][t + 1]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int tok = 2 * (j < 2 ? 1 - part : part) + (j & 1);
        const Frag cf = row_frag(cs + (16 * tok + col) * NS + 16 * (t0 + t) + 8 * g);
#pragma unroll
        for (int a = 0; a < kParts; ++a) in[j] = mma(sf.p[a], cf, in[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) ex[j][wave_id()][lane] = in[j];
    fetch_c(k + 1);
    fetch_x(k + 1);
    update_state<T, NT, PARTS, 1>(s, xf, bs, wt[now], total[now], t0);
    __syncthreads();
    f32x4 y[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (q > part) break;
#pragma unroll
      for (int a = 0; a < kParts; ++a) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          y[j] = mma(xf[0][q], row_frag(lg[a] + (part ? 32 * LS0 + (16 * j + col) * LS1
                                                   : (16 * j + col) * LS0) + 32 * q + 8 * g), y[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int s16 = 16 * (2 * part + j) + col;
      const float ec = exp2_diff(hi[now][s16], lo[now][s16], 0.0f, 0.0f);
      const f32x4 more = ex[j][wave_id() ^ 4][lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[j][i] += decayed(ec, in[2 + j][i] + more[i]);
      // over x, of which every wave has read what it needs
      *reinterpret_cast<typename Elem<T>::Four*>(xs + s16 * XS + 16 * wave + 4 * g) =
          to_four<T>(y[j]);
    }
  }
  __syncthreads();
  XStage y_out;
  y_out.take(xs, XS);
  put_y(y_out, count - 1);
  if (d.fin && where.seg + 1 == sh.segs)
    store_state<VEC>(s[0], d.fin + at.at * size + (uint64_t)at.p0 * N, p, at.rows, N, t0);
}

// ------------------------------------------------------------ gradient

constexpr int kGradThreads = 768;

// Gradients of one chunk, all heads of a split in turn (their sum is dB and
// dC).  S the state that enters the chunk, R the adjoint of the one that
// leaves it, K_{s,r} = dy_s . x_r, G_{s,r} = C_s . B_r, D_{s,r} = e^{cum_s - cum_r}
// (0 for r > s), w_r = e^{cum_Q - cum_r}:
//   dx_r = sum_s (D G)_{s,r} dy_s + w_r R B_r
//   dC_s = sum_r W_{s,r} B_r + sum_h e^{cum_s} S^T dy_s,   W = sum_h D K
//   dB_r = sum_s W_{s,r} C_s + sum_h w_r R^T x_r
//   dla_t = sum_{s >= t > r} (D K G)_{s,r} + sum_{s >= t} C_s . (e^{cum_s} S^T dy_s)
//           + sum_{r < t} B_r . (w_r R^T x_r) + e^{cum_Q} <R, S>
// Every term of dla_t has decays across t in it; only such terms are added up, so that the
// result is as exact where e^{la_t} is small (sums from which larger ones cancel would not
// be).  The first is, column by column, the sum of D K G from row t on, over r < t.
// Wave w of 0..3 holds the columns r = 16 w ... of G, K and W
// and forms dx; wave 4 + 4 e + w holds half e of the entries of dC and dB for the
// tokens 16 w ....  S and R come in fp32; they, D G and W enter the products in two
// bfloat16 parts, so that every gradient is rounded once.  8 x 2048 tokens, 24 heads:
// 154 us for 560 MB, 3.6 TB/s; a copy's rate would give 114, LDS is busy for 65.
template <typename T, int NT, bool VEC>
__global__ __launch_bounds__(kGradThreads) void k_scan_grad(ScanShape sh, ScanGrad a) {
  constexpr int XS = PT + Elem<T>::kPad, NS = NT + Elem<T>::kPad;
  __shared__ __align__(16) T bs[Q * NS];
  __shared__ __align__(16) T cs[Q * NS];
  using Two = Parts<T, 2>;
  constexpr int kParts = Two::kCount;
  // In bfloat16 the tokens of the rounds lie in turn in two places, and S and R, in
  // their parts, in one each: S is replaced while R is read and the other way round, two
  // barriers a round.  In float32 LDS has room for one place, R following S in it.
  constexpr bool kApart = sizeof(T) == 2;
  constexpr int kPlaces = kApart ? 2 : 1;
  __shared__ __align__(16) T x_s[kPlaces][Q * XS];
  __shared__ __align__(16) T dy_s[kPlaces][Q * XS];
  __shared__ __align__(16) T s_s[kPlaces][kParts][PT * NS];
  __shared__ __align__(16) float hi_s[2][Q], lo_s[2][Q], ec_s[2][Q], wt_s[2][Q];
  // of the round at hand and of the one before, whose dla is still to be formed;
  // what is written before a round's barrier, also of the round to come
  __shared__ float us[2][2][Q], vs[2][2][Q], across[2][4][Q], dots[4][8], total[4];
  using Frag = typename Elem<T>::Frag;
  const int wave = wave_id();
  int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  const bool left = wave < 4;  // waves of dx
  const int tile = wave & 3;
  const int P = sh.head_dim, N = sh.d_state;
  const uint32_t bc = blockIdx.x;
  const uint32_t b = bc / sh.chunks, c = bc % sh.chunks;
  const uint32_t grp = blockIdx.y / a.splits, split = blockIdx.y % a.splits;
  const int64_t t0 = (int64_t)c * Q;
  const int n = min((int64_t)Q, (int64_t)sh.len - t0);
  const uint32_t per_group = sh.heads / sh.groups;
  const uint32_t h0 = split * a.heads_per_split;
  const uint32_t hn = min(a.heads_per_split, per_group - h0);

  // Waves 0..3 bring x and dy of a round, the others S and R, two neighbouring tiles of a
  // lane at a time.
  using XStage = Stage<T, Q, PT, 256, VEC>;
  XStage x_next, dy_next;
  constexpr int kPairs = PT * NT / 8 / 512;
  f32x4 s_next[kPairs][2], r_next[kPairs][2];
  if (!left) {
    using NStage = Stage<T, Q, NT, 512, VEC, 256>;
    NStage st, st2;
    st.load((const T*)a.b + b * a.b_batch + t0 * a.b_token + (int64_t)grp * N,
            typename NStage::In(a.b_token, N), n);
    st2.load((const T*)a.c + b * a.c_batch + t0 * a.c_token + (int64_t)grp * N,
             typename NStage::In(a.c_token, N), n);
    st.store(bs, NS);
    st2.store(cs, NS);
  }
  // One of the waves with states, which have less to do, forms dla of the round before;
  // the running sums of the next are left to the wave with least of K.
  constexpr int kFinish = 4, kSums = 3;
  uint32_t lav = 0;  // as loaded: a conversion would wait for it
  const uint32_t la_at =
      lane < n ? lane * (uint32_t)sh.la_token * (uint32_t)sizeof(T) : kAbsent;
  // the loads of round k (head of the split and channel tile)
  auto tokens = [&](const void* base, uint64_t batch, uint64_t token, uint32_t k, XStage& st) {
    const uint32_t h = grp * per_group + h0 + k / sh.ptiles, pt = k % sh.ptiles;
    st.load((const T*)base + b * batch + t0 * token + (int64_t)h * P + pt * PT,
            typename XStage::In(token, min(PT, P - (int)pt * PT)), n);
  };
  // pair i of a lane: row 16 w + col, entries 32 q + 8 g ...
  auto pair = [&](int i, int* w, int* q) {
    *w = (wave - 4 + 8 * i) / (NT / 32);
    *q = (wave - 4 + 8 * i) % (NT / 32);
  };
  auto states = [&](const float* base, uint32_t k, f32x4(&to)[kPairs][2]) {
    const uint32_t h = grp * per_group + h0 + k / sh.ptiles, pt = k % sh.ptiles;
    const Mem m(base + sh.chunk_state((uint64_t)b * sh.heads + h, c, pt));
    const int entries = sh.kept_entries();
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      int w, q;
      pair(i, &w, &q);
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const bool seen = 16 * w + col < P - (int)pt * PT && state_col(2 * q + f, g) < N;
        to[i][f] = __builtin_bit_cast(
            f32x4, m.load16(seen ? kept_at(w, 2 * q + f, lane, entries) : kAbsent));
      }
    }
  };
  auto place_states = [&](T(&to)[kParts][PT * NS], const f32x4(&from)[kPairs][2]) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      int w, q;
      pair(i, &w, &q);
      Two v;
      v.split(from[i][0], from[i][1]);
#pragma unroll
      for (int a = 0; a < kParts; ++a)
        *reinterpret_cast<Frag*>(to[a] + (16 * w + col) * NS + 32 * q + 8 * g) = v.p[a];
    }
  };
  auto fetch = [&](uint32_t k) {
    if (wave == kSums) {
      const uint32_t h = grp * per_group + h0 + k / sh.ptiles;
      lav = Mem((const T*)sh.la + b * sh.la_batch + t0 * sh.la_token + h).load_bits<T>(la_at);
    }
    tokens(a.x, a.x_batch, a.x_token, k, x_next);
    tokens(a.dy, a.dy_batch, a.dy_token, k, dy_next);
  };
  __syncthreads();

  // waves 0..3: tiles (s = 16 j + 4 g + i, r = 16 tile + col) of G and W;
  // the others: (n = state_col(first + t, g) + i, token 16 tile + col) of dC and dB
  constexpr int kOwn = NT / 32;
  const int half_of = left ? 0 : (wave >> 2) - 1, first = half_of * kOwn;
  f32x4 gt[4], wk[4];
  f32x4 dc[kOwn], db[kOwn];
#pragma unroll
  for (int j = 0; j < 4; ++j) gt[j] = wk[j] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < kOwn; ++t) dc[t] = db[t] = f32x4{0, 0, 0, 0};
  if (left) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j >= tile) {
#pragma unroll
        for (int q = 0; q < NT; q += 32)
          gt[j] = mma(row_frag(cs + (16 * j + col) * NS + q + 8 * g),
                      row_frag(bs + (16 * tile + col) * NS + q + 8 * g), gt[j]);
      }
    }
  }
  // out += scale (state in LDS)^T tok for this wave's tokens and entries, and
  // into `to` the products of what was added with the tokens' rows of `rowsn`.
  // Entries lie as in the recurrence's kernels: tiles 2 q and 2 q + 1 together
  // are those of one row access.
  auto sum_state = [&](f32x4(&out)[kOwn], const T(&sr)[kParts][PT * NS], const T* tok,
                       const T* rowsn, float scale, float* to) {
    Frag tf[PT / 32];
#pragma unroll
    for (int q = 0; q < PT / 32; ++q) tf[q] = row_frag(tok + (16 * tile + col) * XS + 32 * q + 8 * g);
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < kOwn; t += 2) {
      __builtin_amdgcn_sched_barrier(0);  // one pair's operands at a time in the registers
      f32x4 acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int q = 0; q < PT / 32; ++q) {
#pragma unroll
        for (int a = 0; a < kParts; ++a) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
            acc[e] = mma(join(state_four(sr[a], NS, 32 * q + 8 * g, first + t + e),
                              state_four(sr[a], NS, 32 * q + 8 * g + 4, first + t + e)), tf[q],
                         acc[e]);
        }
      }
      const Frag row = row_frag(rowsn + (16 * tile + col) * NS + 16 * (first + t) + 8 * g);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const f32x4 rv = half(row, e);
        acc[e] = decayed(scale, acc[e]);
        out[t + e] += acc[e];
        sum += (acc[e][0] * rv[0] + acc[e][1] * rv[1]) + (acc[e][2] * rv[2] + acc[e][3] * rv[3]);
      }
    }
    sum = sum_groups(sum);
    if (g == 0) to[16 * tile + col] = sum;
  };
  // dla of round k, by one wave, from what the waves left in LDS
  float dla = 0.0f;  // token `lane`, summed over the channel tiles of a head
  auto finish = [&](uint32_t k) {
    const int b2 = k & 1, b4 = k & 3;
    float base = 0.0f;
#pragma unroll
    for (int x = 0; x < 8; ++x) base += dots[b4][x];
    const float own = (across[b2][0][lane] + across[b2][1][lane]) +
                      (across[b2][2][lane] + across[b2][3][lane]);
    const float u = us[b2][0][lane] + us[b2][1][lane];
    const float v = vs[b2][0][lane] + vs[b2][1][lane];
    float after = u, before = v;  // sums from the token on, and up to it
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      const float p = __shfl_down(after, x), q = __shfl_up(before, x);
      after += lane + x < 64 ? p : 0.0f;
      before += lane >= x ? q : 0.0f;
    }
    const float upto = __shfl_up(before, 1);
    dla += own + after + (lane ? upto : 0.0f) + decayed(total[b4], base);
    if (k % sh.ptiles + 1 == sh.ptiles) {
      const uint32_t h = grp * per_group + h0 + k / sh.ptiles;
      if (lane < n) ((T*)a.dla)[((uint64_t)b * sh.len + t0 + lane) * sh.heads + h] = (T)dla;
      dla = 0.0f;
    }
  };
  const uint32_t rounds = hn * sh.ptiles;
  // Both kinds of waves run through the same rounds and barriers, each with the
  // registers of its own part only.
  auto run = [&](auto is_left) {
    if constexpr (is_left) {
      fetch(0);
    } else {
      states(a.s_in, 0, s_next);
      states(a.r_in, 0, r_next);
    }
    Cum cum;
    if (is_left && wave == kSums) cum = cumulate(Mem::value<T>(lav));
#pragma unroll 1
    for (uint32_t k = 0; k < rounds; ++k) {
      // addresses are formed anew in every round: kept, they would leave too few registers,
      // and a spilled one waits for all loads under way (155 us for 179)
      asm volatile("" : "+v"(lane));
      col = lane & 15, g = lane >> 4;
      const uint32_t h = grp * per_group + h0 + k / sh.ptiles, pt = k % sh.ptiles;
      const int p0 = pt * PT, rows = min(PT, P - p0), now = k & 1;
      const int place = kApart ? now : 0, at4 = k & 3;
      T *xs = x_s[place], *dys = dy_s[place];
      auto &sr = s_s[0], &rr = s_s[kPlaces - 1];
      float *hi = hi_s[now], *lo = lo_s[now], *ec = ec_s[now], *wt = wt_s[now];
      if constexpr (!kApart) __syncthreads();
      if constexpr (is_left) {
        x_next.store(xs, XS);
        dy_next.store(dys, XS);
      } else {
        place_states(sr, s_next);
      }
      if (is_left && wave == kSums) {
        hi[lane] = cum.hi;
        lo[lane] = cum.lo;
        ec[lane] = cum.e;
        wt[lane] = cum.w;
        if (lane == 0) total[at4] = cum.total;
      }
      __syncthreads();
      if constexpr (!is_left) {
        // <R, S> of the round; then their registers are free for the next one
        f32x4 dot = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
#pragma unroll
          for (int f = 0; f < 2; ++f) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              dot[e] = __builtin_fmaf(r_next[i][f][e], s_next[i][f][e], dot[e]);
          }
        }
        if constexpr (kApart) place_states(rr, r_next);
        if (k + 1 < rounds) {
          states(a.s_in, k + 1, s_next);
          if constexpr (kApart) states(a.r_in, k + 1, r_next);
        }
        const float sum = sum_groups(sum16((dot[0] + dot[1]) + (dot[2] + dot[3])));
        if (lane == 0) dots[at4][wave - 4] = sum;
        if (wave == kFinish && k) finish(k - 1);
      } else {
        if (k + 1 < rounds) fetch(k + 1);
      }
      Two dg[2];  // D G as an operand, summed over s: halves of the chunk
      if constexpr (is_left) {
        const float hr = hi[16 * tile + col], lr = lo[16 * tile + col];
        // of the tokens t = 16 j + 4 g + i, the sum over s >= t of D K G at (s, r)
        float rows16[16], below = 0.0f;
        Frag xf[PT / 32];
  #pragma unroll
        for (int q = 0; q < PT / 32; ++q)
          xf[q] = row_frag(xs + (16 * tile + col) * XS + 32 * q + 8 * g);
        f32x4 weight[4];  // D G, rows 16 j + 4 g + i
  #pragma unroll
        for (int j = 3; j >= 0; --j) {
          f32x4 m = {0, 0, 0, 0}, e = {0, 0, 0, 0};
          if (j >= tile) {
  #pragma unroll
            for (int q = 0; q < PT / 32; ++q)
              m = mma(row_frag(dys + (16 * j + col) * XS + 32 * q + 8 * g), xf[q], m);
            const f32x4 hs = *reinterpret_cast<const f32x4*>(hi + 16 * j + 4 * g);
            const f32x4 ls = *reinterpret_cast<const f32x4*>(lo + 16 * j + 4 * g);
  #pragma unroll
            for (int i = 0; i < 4; ++i) {
              e[i] = exp2_seen(j > tile || 4 * g + i >= col, hs[i], ls[i], hr, lr);
              m[i] *= e[i];
            }
            wk[j] += m;
            e *= gt[j];
            m *= gt[j];
  #pragma unroll
            for (int i = 2; i >= 0; --i) m[i] += m[i + 1];
            below = add_later_groups(m, below);
          }
          weight[j] = e;
  #pragma unroll
          for (int i = 0; i < 4; ++i)
            rows16[4 * j + i] = j > tile || (j == tile && 4 * g + i > col) ? m[i] : 0.0f;
        }
  #pragma unroll
        for (int e = 0; e < 2; ++e) dg[e].split(weight[2 * e], weight[2 * e + 1]);
        across[now][tile][16 * (col >> 2) + 4 * g + (col & 3)] = sums16(rows16);
      } else {
        sum_state(dc, sr, dys, cs, ec[16 * tile + col], us[now][half_of]);
      }
      __syncthreads();
      if constexpr (!kApart) {
        if constexpr (!is_left) {
          place_states(rr, r_next);
          if (k + 1 < rounds) states(a.r_in, k + 1, r_next);
        }
        __syncthreads();
      }
      if constexpr (is_left) {
        const float wr = wt[16 * tile + col];
        Frag bf[NT / 32];
  #pragma unroll
        for (int q = 0; q < NT / 32; ++q)
          bf[q] = row_frag(bs + (16 * tile + col) * NS + 32 * q + 8 * g);
        const Mem dx((T*)a.dx + (((uint64_t)b * sh.len + t0) * sh.heads + h) * P + p0);
        const uint32_t at = (16 * tile + col) * sh.heads * P * (uint32_t)sizeof(T);
  #pragma unroll
        for (int x = 0; x < PT / 16; x += 2) {
          f32x4 acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  #pragma unroll
          for (int q = 0; q < NT / 32; ++q) {
  #pragma unroll
            for (int a = 0; a < kParts; ++a) {
  #pragma unroll
              for (int e = 0; e < 2; ++e)
                acc[e] = mma(row_frag(rr[a] + (16 * (x + e) + col) * NS + 32 * q + 8 * g), bf[q],
                             acc[e]);
            }
          }
  #pragma unroll
          for (int e = 0; e < 2; ++e) acc[e] = decayed(wr, acc[e]);
  #pragma unroll
          for (int j = 0; j < 4; j += 2) {
            if (j + 1 >= tile) {
  #pragma unroll
              for (int e = 0; e < 2; ++e) {
                const Frag dyf = join(col_four(dys, XS, 16 * j + 4 * g, 16 * (x + e)),
                                      col_four(dys, XS, 16 * j + 16 + 4 * g, 16 * (x + e)));
  #pragma unroll
                for (int a = 0; a < kParts; ++a) acc[e] = mma(dyf, dg[j / 2].p[a], acc[e]);
              }
            }
          }
  #pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int pp = 16 * (x + e) + 4 * g;
            dx.store_four<T, VEC>(at + pp * (uint32_t)sizeof(T), acc[e],
                                  16 * tile + col < n ? rows - pp : 0);
          }
        }
      } else {
        sum_state(db, rr, xs, bs, wt[16 * tile + col], vs[now][half_of]);
      }
      if (is_left && wave == kSums && k + 1 < rounds) cum = cumulate(Mem::value<T>(lav));
    }
    __syncthreads();
    if (!is_left && wave == kFinish) finish(rounds - 1);
  };
  if (left)
    run(std::true_type{});
  else
    run(std::false_type{});
  // W to LDS (rows s, columns r), then its products with B and C
  if (left) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float w = wk[j][i];
#pragma unroll
        for (int a = 0; a < kParts; ++a) {
          const T part = (T)w;
          x_s[a][(16 * j + 4 * g + i) * XS + 16 * tile + col] = part;
          w -= (float)part;
        }
      }
  }
  __syncthreads();
  if (left) return;
  const uint64_t row = (((uint64_t)b * sh.len + t0) * sh.groups + grp) * N;
  const uint64_t part = (uint64_t)split * sh.batch * sh.len * sh.groups * N + row;
  const Mem dcm(a.dc_part ? (void*)(a.dc_part + part) : (void*)((T*)a.dc + row));
  const Mem dbm(a.db_part ? (void*)(a.db_part + part) : (void*)((T*)a.db + row));
  Frag wc[kParts][2], wb[kParts][2];
#pragma unroll
  for (int a = 0; a < kParts; ++a) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      wc[a][q] = row_frag(x_s[a] + (16 * tile + col) * XS + 32 * q + 8 * g);
      wb[a][q] = join(col_four(x_s[a], XS, 32 * q + 8 * g, 16 * tile),
                      col_four(x_s[a], XS, 32 * q + 8 * g + 4, 16 * tile));
    }
  }
#pragma unroll
  for (int x = 0; x < kOwn; ++x) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const Frag bf = join(state_four(bs, NS, 32 * q + 8 * g, first + x),
                           state_four(bs, NS, 32 * q + 8 * g + 4, first + x));
      const Frag cf = join(state_four(cs, NS, 32 * q + 8 * g, first + x),
                           state_four(cs, NS, 32 * q + 8 * g + 4, first + x));
#pragma unroll
      for (int a = 0; a < kParts; ++a) {
        dc[x] = mma(bf, wc[a][q], dc[x]);
        db[x] = mma(cf, wb[a][q], db[x]);
      }
    }
    const int nn = state_col(first + x, g);
    const uint32_t at = (16 * tile + col) * sh.groups * N + nn;
    const int some = 16 * tile + col < n ? N - nn : 0;
    if (a.db_part) {
      dcm.store_four<float, VEC>(at * 4, dc[x], some);
      dbm.store_four<float, VEC>(at * 4, db[x], some);
    } else {
      dcm.store_four<T, VEC>(at * (uint32_t)sizeof(T), dc[x], some);
      dbm.store_four<T, VEC>(at * (uint32_t)sizeof(T), db[x], some);
    }
  }
}

// Sum of the splits' parts of dB (blockIdx.y = 0) or dC (1), in their order.
template <typename T>
__global__ __launch_bounds__(256) void k_scan_parts(ScanGrad a, uint64_t count) {
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= count) return;
  const float* p = (blockIdx.y ? a.dc_part : a.db_part) + i;
  float s = p[0];
  for (uint32_t k = 1; k < a.splits; ++k) s += p[k * count];
  ((T*)(blockIdx.y ? a.dc : a.db))[i] = (T)s;
}

// ------------------------------------------------------------ one token

// One served token per row: S = e^{la} S + x B^T in place, y = S C.  Memory
// bound by the state, which is read and written once: 250 rows of 24 heads of
// 64 x 128 in 59.5 us (6.6 TB/s) with part of the states still in the memory-side
// cache, 79 us a call (5 TB/s, a copy's rate) where they are not.  LPR lanes share
// one state row, four entries each, so that loads and stores are whole lines.
template <typename T, int LPR, bool VEC>
__global__ __launch_bounds__(256) void k_scan_step(StepArgs a, uint32_t psplit) {
  constexpr int kRows = 256 / LPR;  // state rows per pass of the workgroup
  const uint32_t ps = blockIdx.x % psplit;
  const uint64_t rh = blockIdx.x / psplit;
  const uint32_t h = rh % a.heads;
  const uint64_t row = rh / a.heads;
  const int P = a.head_dim, N = a.d_state;
  const int n = threadIdx.x % LPR * 4, sub = threadIdx.x / LPR;
  const int64_t slot = a.slots ? (int64_t)a.slots[row] : (int64_t)row;
  T* y = (T*)a.y + (row * a.heads + h) * P;
  if (slot < 0 || slot >= (int64_t)a.pool) {  // an idle row
    for (int p = ps * kRows + sub; p < P; p += psplit * kRows)
      if (n == 0) y[p] = (T)0.0f;
    return;
  }
  const uint32_t g = h / (a.heads / a.groups);
  const T* x = (const T*)a.x + row * a.x_row + (int64_t)h * P;
  const T* bp = (const T*)a.b + row * a.b_row + (int64_t)g * N + n;
  const T* cp = (const T*)a.c + row * a.c_row + (int64_t)g * N + n;
  const float decay = expf(load1((const T*)a.la + row * a.la_row + h));
  f32x4 b, c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    b[i] = n + i < N ? load1(bp + i) : 0.0f;
    c[i] = n + i < N ? load1(cp + i) : 0.0f;
  }
  const Mem s(a.state + ((uint64_t)slot * a.heads + h) * P * N);
  for (int p = ps * kRows + sub; p < P; p += psplit * kRows) {
    f32x4 v = s.load_four<VEC>((p * N + n) * 4, N - n);
    const float xv = load1(x + p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(decay, decay == 0.0f ? 0.0f : v[i], xv * b[i]);
    s.store_four<float, VEC>((p * N + n) * 4, v, N - n);
    float d = (v[0] * c[0] + v[1] * c[1]) + (v[2] * c[2] + v[3] * c[3]);
#pragma unroll
    for (int k = 1; k < LPR; k *= 2) d += __shfl_xor(d, k);
    if (n == 0) y[p] = (T)d;
  }
}

__global__ __launch_bounds__(256) void k_state_copy(const float* from, float* to, uint64_t count) {
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < count;
       i += (uint64_t)gridDim.x * 256)
    to[i] = from ? from[i] : 0.0f;
}

template <typename T, int NT, bool VEC, int PARTS, int HB, int EW>
hipError_t states(const ScanShape& sh, const ScanDir* d, int nd, bool main, hipStream_t s) {
  const ScanDir &d0 = d[0], &d1 = d[nd - 1];
  const dim3 grid(sh.batch * sh.segs * (sh.heads * sh.ptiles / HB), (sh.d_state + NT - 1) / NT, nd);
  if (sh.segs > 1) {
    k_scan_states<T, NT, VEC, PARTS, HB, EW><<<grid, 256 * EW, 0, s>>>(sh, d0, d1, true);
    if (hipError_t e = hipGetLastError()) return e;
    if (sh.joined) {
      const uint32_t blocks = (sh.head_dim * sh.d_state + 255) / 256;
      k_scan_join<<<dim3(blocks * sh.batch * sh.heads, 1, nd), 256, 0, s>>>(sh, d0, d1);
      if (hipError_t e = hipGetLastError()) return e;
    }
  }
  if (!main) return hipSuccess;
  k_scan_states<T, NT, VEC, PARTS, HB, EW><<<grid, 256 * EW, 0, s>>>(sh, d0, d1, false);
  return hipGetLastError();
}
// A gradient's states: the two halves of a long state's entries need nothing of each
// other, so in bfloat16 they go to workgroups of four waves, three on a compute unit.  384
// tiles of 32 chunks: 126 us for 403 MB of states (108 at a copy's rate, with what is read);
// while states were half that size, 96, and with eight waves for the whole state 109.
template <typename T, int NT, bool VEC, int PARTS>
hipError_t grad_states(const ScanShape& sh, const ScanDir* d, int nd, hipStream_t s) {
  if constexpr (sizeof(T) == 2 && VEC && NT == 128)
    return states<T, 64, VEC, PARTS, 1, 1>(sh, d, nd, true, s);
  else
    return states<T, NT, VEC, PARTS, 1, 2>(sh, d, nd, true, s);
}
template <typename T, int NT, bool VEC, int PARTS>
hipError_t outputs(const ScanShape& sh, const ScanDir& d, const ScanOut& o, hipStream_t s) {
  hipError_t e;
  if constexpr (sizeof(T) == 2 && VEC)
    e = sh.tiles == 2 ? states<T, NT, VEC, PARTS, 2, 1>(sh, &d, 1, false, s)
                      : states<T, NT, VEC, PARTS, 1, 2>(sh, &d, 1, false, s);
  else
    e = states<T, NT, VEC, PARTS, 1, 2>(sh, &d, 1, false, s);
  if (e) return e;
  k_scan_out<T, NT, VEC, PARTS>
      <<<sh.batch * sh.segs * sh.heads * sh.ptiles, 512, 0, s>>>(sh, d, o);
  return hipGetLastError();
}
// Weighted inputs in three parts where a state is an output, otherwise in two: see Parts.
#define FESC_SCAN_PARTS(CALL)              \
  if constexpr (sizeof(T) == 2 && VEC) {   \
    if (!sh.exact) return CALL(2);         \
  }                                        \
  return CALL(3)
template <typename T, int NT, bool VEC>
hipError_t states(const ScanShape& sh, const ScanDir* d, int nd, hipStream_t s) {
#define FORM(PARTS) (grad_states<T, NT, VEC, PARTS>(sh, d, nd, s))
  FESC_SCAN_PARTS(FORM);
#undef FORM
}
template <typename T, int NT, bool VEC>
hipError_t outputs(const ScanShape& sh, const ScanDir& d, const ScanOut& o, hipStream_t s) {
#define FORM(PARTS) (outputs<T, NT, VEC, PARTS>(sh, d, o, s))
  FESC_SCAN_PARTS(FORM);
#undef FORM
}

// One instance per element type, padded state size and alignment.
#define FESC_SCAN_N(T, SH, CALL)                                                 \
  ((SH).d_state <= 64 ? ((SH).vec ? CALL(T, 64, true) : CALL(T, 64, false))      \
                      : ((SH).vec ? CALL(T, 128, true) : CALL(T, 128, false)))
#define FESC_SCAN_CASES(DTYPE, SH, CALL) \
  ((DTYPE) == FESC_BF16 ? FESC_SCAN_N(__bf16, SH, CALL) : FESC_SCAN_N(float, SH, CALL))

}  // namespace

hipError_t launch_scan_states(uint32_t dtype, const ScanShape& sh, const ScanDir* d, int nd,
                              hipStream_t s) {
#define CALL(T, NT, VEC) states<T, NT, VEC>(sh, d, nd, s)
  return FESC_SCAN_CASES(dtype, sh, CALL);
#undef CALL
}

hipError_t launch_scan_out(uint32_t dtype, const ScanShape& sh, const ScanDir& d,
                           const ScanOut& o, hipStream_t s) {
#define CALL(T, NT, VEC) outputs<T, NT, VEC>(sh, d, o, s)
  return FESC_SCAN_CASES(dtype, sh, CALL);
#undef CALL
}

hipError_t launch_scan_grad(uint32_t dtype, const ScanShape& sh, const ScanGrad& g,
                            hipStream_t s) {
  const dim3 grid(sh.batch * sh.chunks, sh.groups * g.splits);
#define CALL(T, NT, VEC) (k_scan_grad<T, NT, VEC><<<grid, kGradThreads, 0, s>>>(sh, g), hipGetLastError())
  hipError_t e = FESC_SCAN_CASES(dtype, sh, CALL);
#undef CALL
  if (e || g.splits == 1) return e;
  const uint64_t count = (uint64_t)sh.batch * sh.len * sh.groups * sh.d_state;
  const dim3 pgrid((uint32_t)((count + 255) / 256), 2);
  if (dtype == FESC_BF16)
    k_scan_parts<__bf16><<<pgrid, 256, 0, s>>>(g, count);
  else
    k_scan_parts<float><<<pgrid, 256, 0, s>>>(g, count);
  return hipGetLastError();
}

hipError_t launch_scan_step(uint32_t dtype, const StepArgs& a, hipStream_t s) {
  const uint32_t lpr = a.d_state <= 64 ? 16 : 32, rows = 256 / lpr;
  const uint32_t passes = (a.head_dim + rows - 1) / rows;
  const uint64_t heads = (uint64_t)a.rows * a.heads;
  // A head's passes (8 here) go to as many workgroups as make three on each compute
  // unit.  24 heads in one, four, eight workgroups each: 6.1, 4.2, 3.9 us; 192: 8.2,
  // 6.2, 7.2; 480: 9.8, 10.1, 12.3; 6000: 62, 63, 92.
  const uint32_t psplit =
      (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(passes, heads ? 768 / heads : 1));
  const uint32_t grid = (uint32_t)(heads * psplit);
#define STEP(T, LPR)                                                 \
  if (a.vec)                                                         \
    k_scan_step<T, LPR, true><<<grid, 256, 0, s>>>(a, psplit);       \
  else                                                               \
    k_scan_step<T, LPR, false><<<grid, 256, 0, s>>>(a, psplit)
  if (dtype == FESC_BF16) {
    if (lpr == 16) {
      STEP(__bf16, 16);
    } else {
      STEP(__bf16, 32);
    }
  } else {
    if (lpr == 16) {
      STEP(float, 16);
    } else {
      STEP(float, 32);
    }
  }
#undef STEP
  return hipGetLastError();
}

hipError_t launch_state_copy(const float* from, float* to, uint64_t count, hipStream_t s) {
  const uint32_t grid = (uint32_t)std::min<uint64_t>((count + 255) / 256, 1u << 16);
  k_state_copy<<<grid, 256, 0, s>>>(from, to, count);
  return hipGetLastError();
}

}  // namespace fesc
