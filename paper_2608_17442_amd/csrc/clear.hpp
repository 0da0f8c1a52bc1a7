// The block in the clear: arguments of the recurrence and norm kernels
// (clear_scan.hip, clear_norm.hip), filled in and checked by clear.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fesc.h"

namespace fesc {

constexpr uint32_t kChunk = 64;   // tokens whose decay matrix is formed at once
constexpr uint32_t kPTile = 64;   // channels of one head held by one workgroup
constexpr uint32_t kMaxState = 128;

// One direction of the recurrence over the sequence.  Forward: u = x, v = B,
// states move from the first chunk to the last.  Reverse (the adjoint of the
// states): u = dy, v = C, from the last chunk to the first.
struct ScanDir {
  const void* u;
  const void* v;
  int64_t u_token, u_batch, v_token, v_batch;
  const float* init;   // [b][h][P][N] or null (zero)
  float* fin;          // [b][h][P][N] or null
  float* chunk_states;  // [b][h][chunk][channel tile][kept rows * entries] or null: the
                        // state that enters each chunk, in the order in which lanes hold it
  float* seg_states;   // [b][h][segment][P][N] or null (one segment)
  float* seg_decay;    // [b][h][segment]
  bool reverse;
};

struct ScanShape {
  uint32_t batch, len, heads, head_dim, groups, d_state;
  uint32_t chunks;      // ceil(len / kChunk)
  uint32_t seg_chunks;  // chunks per segment
  uint32_t segs;
  bool joined;          // the summaries of many segments are joined by a kernel of its own
  uint32_t ptiles;      // ceil(head_dim / kPTile)
  uint32_t tiles;       // channel tiles in one workgroup of the segments' own pass: 1, or 2
                        // (aligned bfloat16)
  const void* la;
  int64_t la_token, la_batch;
  bool vec;    // every row of every array starts at a multiple of 16 bytes

  // Entries of a row and rows of a channel tile that chunk states have room for (whole
  // tiles of the matrix instructions), and where that of a channel tile begins
  // (head: batch * heads + head).
  __host__ __device__ uint32_t kept_entries() const { return (d_state + 31) / 32 * 32; }
  __host__ __device__ uint32_t kept_rows() const {
    return ptiles > 1 ? kPTile : (head_dim + 15) / 16 * 16;
  }
  __host__ __device__ uint64_t chunk_state(uint64_t head, uint32_t chunk, uint32_t ptile) const {
    return ((head * chunks + chunk) * ptiles + ptile) * kept_rows() * kept_entries();
  }
  bool exact;  // a state is an output
};

struct ScanOut {  // outputs of a forward scan beside the final state
  const void* c;
  int64_t c_token, c_batch;
  void* y;
};

struct ScanGrad {
  const void *x, *b, *c, *dy;
  int64_t x_token, x_batch, b_token, b_batch, c_token, c_batch, dy_token, dy_batch;
  const float *s_in, *r_in;  // chunk states of the two directions
  void *dx, *dla, *db, *dc;
  float *db_part, *dc_part;  // [split][b][t][G][N] when heads are split, else null
  uint32_t splits, heads_per_split;
};

struct StepArgs {
  const void *x, *la, *b, *c;
  int64_t x_row, la_row, b_row, c_row;
  float* state;
  const int32_t* slots;
  void* y;
  uint32_t rows, pool, heads, head_dim, groups, d_state;
  bool vec;  // state rows start at multiples of 16 bytes
};

struct NormArgs {
  uint64_t rows;
  uint32_t width;
  float eps;
  const void *a, *b, *c;   // gated: m, x, z; residual: o, r
  int64_t a_row, b_row, c_row;
  const void *k, *w;       // skip or scale; weight
  void *u, *r_new;
  // backward
  const void *du, *dr_new;
  int64_t du_row, dr_row;
  void *da, *db, *dc, *dk, *dw;
  float* part;             // [blocks][2][width]
  uint32_t blocks;
  bool vec;
};

// Every state pass of a call: the segments' own states and their join (only
// when there are several), then the chunk states and final states.
hipError_t launch_scan_states(uint32_t dtype, const ScanShape& sh, const ScanDir* dirs, int ndirs,
                              hipStream_t s);
hipError_t launch_scan_out(uint32_t dtype, const ScanShape& sh, const ScanDir& dir,
                           const ScanOut& out, hipStream_t s);
hipError_t launch_scan_grad(uint32_t dtype, const ScanShape& sh, const ScanGrad& g, hipStream_t s);
hipError_t launch_scan_step(uint32_t dtype, const StepArgs& a, hipStream_t s);
hipError_t launch_state_copy(const float* from, float* to, uint64_t count, hipStream_t s);

hipError_t launch_norm(uint32_t dtype, bool gated, const NormArgs& a, hipStream_t s);
hipError_t launch_norm_grad(uint32_t dtype, bool gated, const NormArgs& a, hipStream_t s);
// Workgroups of the gradient kernel, each with a row of partial sums.
uint32_t norm_grad_blocks(uint64_t rows, uint32_t width, bool vec);

}  // namespace fesc
