// C entry points of the block in the clear: argument checks, workspace
// layout, and the rules that split the work (kernels: clear_scan.hip,
// clear_norm.hip).
#include "clear.hpp"

#include <algorithm>
#include <cmath>

#include "fesc_internal.hpp"

using namespace fesc;

namespace {

hipStream_t S(void* stream) { return reinterpret_cast<hipStream_t>(stream); }

constexpr uint64_t kMaxStride = 1ull << 40;
// A chunk's rows lie within 2^31 bytes of its first one.
constexpr uint64_t kMaxTokenStride = 1ull << 22;
// A launch counts its work items in 32 bits.
constexpr uint64_t kMaxGrid256 = 1ull << 24, kMaxGrid512 = 1ull << 23, kMaxGrid1024 = 1ull << 22;

uint32_t elem_bytes(uint32_t dtype) { return dtype == FESC_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }

int check_scan(const fesc_clear_scan_desc* d) {
  if (!d) return fail(FESC_ERR_ARG, "null descriptor");
  if (d->dtype != FESC_F32 && d->dtype != FESC_BF16)
    return fail(FESC_ERR_ARG, "dtype: float32 or bfloat16");
  if (d->heads == 0 || d->heads > 4096 || d->groups == 0 || d->heads % d->groups)
    return fail(FESC_ERR_ARG, "heads: 1..4096 and a multiple of groups");
  if (d->head_dim == 0 || d->head_dim > 4096) return fail(FESC_ERR_ARG, "head_dim: 1..4096");
  if (d->d_state == 0 || d->d_state > kMaxState) return fail(FESC_ERR_ARG, "d_state: 1..128");
  for (uint64_t s : {d->x_batch, d->la_batch, d->b_batch, d->c_batch, d->dy_batch})
    if (s > kMaxStride) return fail(FESC_ERR_ARG, "batch strides: at most 2^40");
  for (uint64_t s : {d->x_token, d->la_token, d->b_token, d->c_token, d->dy_token})
    if (s > kMaxTokenStride) return fail(FESC_ERR_ARG, "token strides: at most 2^22");
  if (d->heads * d->head_dim > kMaxTokenStride || d->groups * d->d_state > kMaxTokenStride)
    return fail(FESC_ERR_ARG, "heads * head_dim: at most 2^22");
  return FESC_OK;
}

// Rows of 16 bytes: base and strides, in elements, are multiples of them.
struct Rows {
  uint32_t per;  // elements in 16 bytes
  bool ok = true;
  explicit Rows(uint32_t dtype) : per(16 / elem_bytes(dtype)) {}
  Rows& add(const void* p, uint64_t s0 = 0, uint64_t s1 = 0) {
    ok = ok && aligned(p, 16) && s0 % per == 0 && s1 % per == 0;
    return *this;
  }
  Rows& len(uint64_t n) {
    ok = ok && n % per == 0;
    return *this;
  }
};

// How a pass over the sequence is cut.  A workgroup carries the states of its
// channel tiles from chunk to chunk; of the tiles there are
// batch * heads * (directions that run at once), and 256 compute units take one
// or, at some 1.75 times the time of a chunk, two workgroups each (one in
// float32, whose LDS tiles are twice the size).
//  - Many tiles: each takes its sequence as a whole, eight waves, one launch.
//  - Otherwise segments of whole chunks; the price is a pass before, in which x and
//    B are read for the segments' own states, and their join.  Two workgroups a
//    unit where segments of six chunks remain, else one, two chunks at least.
//  - Long sequences: two a unit, and the pass before in workgroups of two tiles (four
//    waves), which share what is read of B.
// Measured with 24 heads of 64, state 128, bfloat16, in us, forward (in brackets:
// segments; the rule takes the lowest of a line or one within 3 % of it):
//    tiles x chunks   whole   one a unit   two a unit   four (two at once), pairs before
//     24 x 32           89       34 (10)      -            -
//     48 x 32           89       45 (5)       51 (10)      -
//     96 x 32           87       75 (2)       60 (5)       64 (10)
//    144 x 32           87        -           80 (3)       87 (7)
//    168 x 32           87        -           81 (3)       97 (6)
//    192 x 32           89        -          113 (2)       97 (5)
//     24 x 128         337       74 (10)      67 (21)      68 (42)
//     48 x 128         337      125 (5)      104 (10)     109 (21)
//     96 x 128         336      270 (2)      182 (5)      170 (10)
//    144 x 128         342        -          274 (3)      249 (7)
//    192 x 128         343        -          402 (2)      321 (5)
//     24 x 782           -      337 (10)     269 (21)     254 (42)
// The same rules for a state of 64 (1 x 2048 tokens 27.6 in 10, best 27.1; 8 x 2048 74, 73;
// 1 x 50001 201 in 42), rows at any alignment (8 x 1581, state 33: 83 whole, best 82;
// 13 x 1827, 20 heads of 100: 355 whole) and float32 (one a unit: 24 x 32 63 in 10;
// 48 x 128 308 in 5; 96 x 32 189 in 2, where 10 would take 169).
// The gradient's pass carries states only, in both directions, so that a cut doubles
// its work; of its workgroups 384 tiles' fit at once (whole gradient call, tiles of
// both directions, segments in brackets):
//     48 x 32           76       63 (5)      63 (8)
//     96 x 16           55       60 (4)      72 (8)
//     96 x 32           89       89 (4)     100 (8)
//    144 x 32          119      138 (3)     152 (8)
//     48 x 128         242      180 (5)     177 (8)
//     96 x 128         353      332 (4)     335 (8)
//     48 x 256         509      357 (5)     333 (8)
//    192 x 128         596      640 (4)     658 (8)
constexpr uint64_t kUnits = 256;
constexpr uint64_t kWholeTiles = 171, kWholeTilesGrad = 96;  // whole from here on
constexpr uint64_t kGradTiles = 384;
constexpr uint64_t kTwoChunks = 2 * kUnits * 6;      // tiles * chunks for two a unit
constexpr uint64_t kPairChunks = 8192;               // tiles * chunks for pairs
constexpr uint64_t kPairTiles = 256;
// Up to this many segments each workgroup adds up the summaries before its own
// (segs / 2 states read on average); more go through the join kernel (each read
// and written once, a launch more).  24 tiles x 32 chunks in 3 segments: 54.6 us
// against 56.1 with the kernel; 5: 40.8, 42.5; 6: 38.3, 39.5; 8: 37.0, 34.0.  96 tiles:
// 5: 60.1, 63.9; 6: 74.2, 80.4; 8: 72.1, 65.7.
constexpr uint32_t kJoinedSegs = 6;
ScanShape shape_of(const fesc_clear_scan_desc* d, int dirs) {
  ScanShape s{};
  s.batch = d->batch;
  s.len = d->len;
  s.heads = d->heads;
  s.head_dim = d->head_dim;
  s.groups = d->groups;
  s.d_state = d->d_state;
  s.la_token = d->la_token;
  s.la_batch = d->la_batch;
  s.chunks = (uint32_t)(((uint64_t)d->len + kChunk - 1) / kChunk);
  s.ptiles = (d->head_dim + kPTile - 1) / kPTile;
  const uint64_t tiles = (uint64_t)d->batch * d->heads * s.ptiles * dirs;
  const bool pairs = d->dtype == FESC_BF16 && d->heads / d->groups * s.ptiles % 2 == 0;
  uint64_t segs = 1;
  s.tiles = 1;
  const uint64_t work = tiles * s.chunks;
  if (tiles && dirs == 2) {
    if (tiles < kWholeTilesGrad)
      segs = std::min<uint64_t>((d->dtype == FESC_BF16 ? kGradTiles : kUnits) / tiles, s.chunks / 4);
  } else if (tiles && pairs && tiles < kPairTiles && work >= kPairChunks) {
    s.tiles = 2;
    segs = 2 * kUnits / (tiles / 2);
  } else if (tiles && tiles < kWholeTiles) {
    if (d->dtype == FESC_BF16 && work >= kTwoChunks)
      segs = 2 * kUnits / tiles;
    else
      segs = std::min<uint64_t>(kUnits / tiles, s.chunks / 2);
  }
  segs = std::max<uint64_t>(1, segs);
  s.seg_chunks = (uint32_t)((s.chunks + segs - 1) / segs);
  s.segs = s.chunks ? (s.chunks + s.seg_chunks - 1) / s.seg_chunks : 1;
  s.joined = s.segs > kJoinedSegs;
  return s;
}

// Heads of a group in turn in one workgroup of the gradient kernel (one on a
// unit); split over workgroups, whose parts of dB and dC are added up, where
// chunks alone leave units idle.  Whole gradient call, 24 heads, in us: 32 chunks in
// 4, 8, 12 splits 71, 64, 74; 64 in 2, 4, 8: 111, 91, 100; 128 in 1, 2, 4: 183, 148,
// 167; 256 in 1, 2: 353, 377.
void split_heads(const ScanShape& s, uint32_t* splits, uint32_t* per) {
  const uint32_t heads = s.heads / s.groups;
  const uint64_t groups = (uint64_t)s.batch * s.chunks * s.groups;
  const uint64_t want = std::min<uint64_t>(heads, std::max<uint64_t>(1, groups ? kUnits / groups : 1));
  *per = (uint32_t)((heads + want - 1) / want);
  *splits = (heads + *per - 1) / *per;
}

uint64_t state_count(const ScanShape& s) {
  return (uint64_t)s.batch * s.heads * s.head_dim * s.d_state;
}

// The workspace, laid out or only measured (base null).
struct Space {
  char* base;
  size_t used = 0;
  explicit Space(void* p) : base((char*)p) {}
  template <typename T>
  T* take(uint64_t count, size_t bytes = sizeof(T)) {
    char* p = base ? base + used : nullptr;
    used += round_up(count * bytes);
    return reinterpret_cast<T*>(p);
  }
};

void seg_space(Space& w, const ScanShape& s, ScanDir* d) {
  if (s.segs == 1) return;
  d->seg_states = w.take<float>(state_count(s) * s.segs);
  d->seg_decay = w.take<float>((uint64_t)s.batch * s.heads * s.segs);
}

void grad_space(Space& w, const ScanShape& s, ScanDir* dir, ScanGrad* g) {
  for (int k = 0; k < 2; ++k) {
    seg_space(w, s, dir + k);
    dir[k].chunk_states = w.take<float>(s.chunk_state((uint64_t)s.batch * s.heads, 0, 0));
  }
  split_heads(s, &g->splits, &g->heads_per_split);
  if (g->splits > 1) {
    const uint64_t n = (uint64_t)s.batch * s.len * s.groups * s.d_state * g->splits;
    g->db_part = w.take<float>(n);
    g->dc_part = w.take<float>(n);
  }
}

// The launches of a call that its sizes alone bound: segments and their join are cut
// for few tiles (kUnits), parts of dB and dC for few chunks.
int check_grid(const ScanShape& s, bool backward) {
  if ((uint64_t)s.batch * s.heads * s.ptiles * s.segs >= kMaxGrid512 ||
      (backward && (uint64_t)s.batch * s.chunks >= kMaxGrid1024))
    return fail(FESC_ERR_ARG, "batch * len * heads too large for one call");
  return FESC_OK;
}

int check_workspace(const void* p, size_t have, size_t need) {
  if (have < need) return fail(FESC_ERR_ARG, "workspace too small");
  if (need && !p) return fail(FESC_ERR_ARG, "null workspace");
  if (!aligned(p, 16)) return fail(FESC_ERR_ARG, "workspace: not aligned to 16 bytes");
  return FESC_OK;
}

int check_norm(const fesc_clear_norm_desc* d) {
  if (!d) return fail(FESC_ERR_ARG, "null descriptor");
  if (d->dtype != FESC_F32 && d->dtype != FESC_BF16)
    return fail(FESC_ERR_ARG, "dtype: float32 or bfloat16");
  if (d->width == 0 || d->width > 16384) return fail(FESC_ERR_ARG, "width: 1..16384");
  if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return fail(FESC_ERR_ARG, "eps: positive");
  for (uint64_t s : {d->m_row, d->x_row, d->z_row, d->o_row, d->r_row, d->du_row, d->dr_row})
    if (s > kMaxStride) return fail(FESC_ERR_ARG, "stride too large");
  if (d->rows > 1ull << 40) return fail(FESC_ERR_ARG, "rows: at most 2^40");
  return FESC_OK;
}

NormArgs norm_args(const fesc_clear_norm_desc* d, bool gated, const void* a, const void* b,
                   const void* c, const void* k, const void* w) {
  NormArgs n{};
  n.rows = d->rows;
  n.width = d->width;
  n.eps = d->eps;
  n.a = a;
  n.b = b;
  n.c = c;
  n.k = k;
  n.w = w;
  n.a_row = gated ? d->m_row : d->o_row;
  n.b_row = gated ? d->x_row : d->r_row;
  n.c_row = gated ? d->z_row : 0;
  n.du_row = d->du_row;
  n.dr_row = d->dr_row;
  return n;
}

bool norm_vec(const fesc_clear_norm_desc* d, const NormArgs& n) {
  Rows r(d->dtype);
  // a lane's unit is 8 channels in either type
  return d->width % 8 == 0 && r.add(n.a, n.a_row).add(n.b, n.b_row).add(n.c, n.c_row)
      .add(n.k, 0).add(n.w, 0).add(n.u, 0).add(n.r_new, 0).add(n.du, n.du ? n.du_row : 0)
      .add(n.dr_new, n.dr_new ? n.dr_row : 0).add(n.da, 0).add(n.db, 0).add(n.dc, 0).ok;
}

int norm_bwd(const fesc_clear_norm_desc* d, bool gated, NormArgs n, void* workspace,
             size_t workspace_bytes, void* stream) {
  size_t need;
  if (int rc = fesc_clear_norm_workspace(d, &need)) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
  n.part = reinterpret_cast<float*>(workspace);
  n.vec = norm_vec(d, n);
  n.blocks = norm_grad_blocks(n.rows, n.width, n.vec);
  return hip_check(launch_norm_grad(d->dtype, gated, n, S(stream)), "norm gradient");
}

}  // namespace

extern "C" {

int fesc_clear_scan_workspace(const fesc_clear_scan_desc* d, int backward, size_t* bytes) {
  if (int rc = check_scan(d)) return rc;
  if (!bytes) return fail(FESC_ERR_ARG, "null argument");
  const ScanShape s = shape_of(d, backward ? 2 : 1);
  Space w(nullptr);
  ScanDir dir[2] = {};
  ScanGrad g{};
  if (backward)
    grad_space(w, s, dir, &g);
  else
    seg_space(w, s, dir);
  *bytes = w.used;
  return FESC_OK;
}

int fesc_clear_scan(const fesc_clear_scan_desc* d, const void* x, const void* la, const void* B,
                    const void* C, const float* h0, void* y, float* hT, void* workspace,
                    size_t workspace_bytes, void* stream) {
  if (int rc = check_scan(d)) return rc;
  ScanShape s = shape_of(d, 1);
  if (int rc = check_grid(s, false)) return rc;
  if (d->batch == 0) return FESC_OK;
  if (d->len == 0)
    return hT ? hip_check(launch_state_copy(h0, hT, state_count(s), S(stream)), "scan") : FESC_OK;
  if (!x || !la || !B || !C || !y) return fail(FESC_ERR_ARG, "null buffer");
  ScanDir dir{};
  Space w(workspace);
  seg_space(w, s, &dir);
  if (int rc = check_workspace(workspace, workspace_bytes, w.used)) return rc;
  s.la = la;
  s.vec = Rows(d->dtype).add(x, d->x_token, d->x_batch).add(B, d->b_token, d->b_batch)
              .add(C, d->c_token, d->c_batch).add(h0).add(hT).add(y).len(d->head_dim)
              .len(d->d_state).ok;
  if (!s.vec) s.tiles = 1;
  s.exact = hT != nullptr;
  dir.u = x;
  dir.v = B;
  dir.u_token = d->x_token;
  dir.u_batch = d->x_batch;
  dir.v_token = d->b_token;
  dir.v_batch = d->b_batch;
  dir.init = h0;
  dir.fin = hT;
  const ScanOut out{C, (int64_t)d->c_token, (int64_t)d->c_batch, y};
  return hip_check(launch_scan_out(d->dtype, s, dir, out, S(stream)), "scan");
}

int fesc_clear_scan_bwd(const fesc_clear_scan_desc* d, const void* x, const void* la,
                        const void* B, const void* C, const float* h0, const void* dy,
                        const float* dhT, void* dx, void* dla, void* db, void* dc, float* dh0,
                        void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_scan(d)) return rc;
  ScanShape s = shape_of(d, 2);
  if (int rc = check_grid(s, true)) return rc;
  if (d->batch == 0) return FESC_OK;
  if (d->len == 0)
    return dh0 ? hip_check(launch_state_copy(dhT, dh0, state_count(s), S(stream)), "scan gradient")
               : FESC_OK;
  if (!x || !la || !B || !C || !dy || !dx || !dla || !db || !dc)
    return fail(FESC_ERR_ARG, "null buffer");
  ScanDir dir[2] = {};
  ScanGrad g{};
  Space w(workspace);
  grad_space(w, s, dir, &g);
  if (int rc = check_workspace(workspace, workspace_bytes, w.used)) return rc;
  s.la = la;
  s.vec = Rows(d->dtype).add(x, d->x_token, d->x_batch).add(B, d->b_token, d->b_batch)
              .add(C, d->c_token, d->c_batch).add(dy, d->dy_token, d->dy_batch).add(h0).add(dhT)
              .add(dh0).add(dx).add(db).add(dc).len(d->head_dim).len(d->d_state).ok;
  if (!s.vec) s.tiles = 1;
  s.exact = dh0 != nullptr;
  dir[0].u = x;
  dir[0].v = B;
  dir[0].u_token = d->x_token;
  dir[0].u_batch = d->x_batch;
  dir[0].v_token = d->b_token;
  dir[0].v_batch = d->b_batch;
  dir[0].init = h0;
  dir[1].u = dy;
  dir[1].v = C;
  dir[1].u_token = d->dy_token;
  dir[1].u_batch = d->dy_batch;
  dir[1].v_token = d->c_token;
  dir[1].v_batch = d->c_batch;
  dir[1].init = dhT;
  dir[1].fin = dh0;
  dir[1].reverse = true;
  if (int rc = hip_check(launch_scan_states(d->dtype, s, dir, 2, S(stream)), "scan gradient"))
    return rc;
  g.x = x;
  g.b = B;
  g.c = C;
  g.dy = dy;
  g.x_token = d->x_token;
  g.x_batch = d->x_batch;
  g.b_token = d->b_token;
  g.b_batch = d->b_batch;
  g.c_token = d->c_token;
  g.c_batch = d->c_batch;
  g.dy_token = d->dy_token;
  g.dy_batch = d->dy_batch;
  g.s_in = dir[0].chunk_states;
  g.r_in = dir[1].chunk_states;
  g.dx = dx;
  g.dla = dla;
  g.db = db;
  g.dc = dc;
  return hip_check(launch_scan_grad(d->dtype, s, g, S(stream)), "scan gradient");
}

int fesc_clear_scan_step(const fesc_clear_scan_desc* d, const void* x, const void* la,
                         const void* B, const void* C, float* state, uint32_t pool,
                         const int32_t* slots, void* y, void* stream) {
  if (int rc = check_scan(d)) return rc;
  if ((uint64_t)d->batch * d->heads >= kMaxGrid256)
    return fail(FESC_ERR_ARG, "batch * heads too large for one call");
  if (!slots && pool < d->batch) return fail(FESC_ERR_ARG, "pool: fewer states than rows");
  if (d->batch == 0) return FESC_OK;
  if (!x || !la || !B || !C || !y || (!state && pool)) return fail(FESC_ERR_ARG, "null buffer");
  StepArgs a{};
  a.x = x;
  a.la = la;
  a.b = B;
  a.c = C;
  a.x_row = d->x_batch;
  a.la_row = d->la_batch;
  a.b_row = d->b_batch;
  a.c_row = d->c_batch;
  a.state = state;
  a.slots = slots;
  a.y = y;
  a.rows = d->batch;
  a.pool = pool;
  a.heads = d->heads;
  a.head_dim = d->head_dim;
  a.groups = d->groups;
  a.d_state = d->d_state;
  a.vec = d->d_state % 4 == 0 && aligned(state, 16);
  return hip_check(launch_scan_step(d->dtype, a, S(stream)), "scan step");
}

int fesc_clear_norm_gated(const fesc_clear_norm_desc* d, const void* m, const void* x,
                          const void* z, const void* skip, const void* w, void* u, void* stream) {
  if (int rc = check_norm(d)) return rc;
  if (d->rows == 0) return FESC_OK;
  if (!m || !x || !z || !skip || !w || !u) return fail(FESC_ERR_ARG, "null buffer");
  NormArgs n = norm_args(d, true, m, x, z, skip, w);
  n.u = u;
  n.vec = norm_vec(d, n);
  return hip_check(launch_norm(d->dtype, true, n, S(stream)), "gated norm");
}

int fesc_clear_norm_residual(const fesc_clear_norm_desc* d, const void* o, const void* r,
                             const void* scale, const void* w, void* r_new, void* u,
                             void* stream) {
  if (int rc = check_norm(d)) return rc;
  if (d->rows == 0) return FESC_OK;
  if (!o || !r || !scale || !w || !r_new || !u) return fail(FESC_ERR_ARG, "null buffer");
  NormArgs n = norm_args(d, false, o, r, nullptr, scale, w);
  n.u = u;
  n.r_new = r_new;
  n.vec = norm_vec(d, n);
  return hip_check(launch_norm(d->dtype, false, n, S(stream)), "residual norm");
}

int fesc_clear_norm_workspace(const fesc_clear_norm_desc* d, size_t* bytes) {
  if (int rc = check_norm(d)) return rc;
  if (!bytes) return fail(FESC_ERR_ARG, "null argument");
  // unaligned rows run in more workgroups than aligned ones
  *bytes = round_up((size_t)norm_grad_blocks(d->rows, d->width, false) * 2 * d->width *
                    sizeof(float));
  return FESC_OK;
}

int fesc_clear_norm_gated_bwd(const fesc_clear_norm_desc* d, const void* m, const void* x,
                              const void* z, const void* skip, const void* w, const void* du,
                              void* dm, void* dx, void* dz, void* dskip, void* dw,
                              void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_norm(d)) return rc;
  if (!skip || !w || !dskip || !dw || (d->rows && (!m || !x || !z || !du || !dm || !dx || !dz)))
    return fail(FESC_ERR_ARG, "null buffer");
  NormArgs n = norm_args(d, true, m, x, z, skip, w);
  n.du = du;
  n.da = dm;
  n.db = dx;
  n.dc = dz;
  n.dk = dskip;
  n.dw = dw;
  return norm_bwd(d, true, n, workspace, workspace_bytes, stream);
}

int fesc_clear_norm_residual_bwd(const fesc_clear_norm_desc* d, const void* o, const void* r,
                                 const void* scale, const void* w, const void* du,
                                 const void* dr_new, void* d_o, void* dr, void* dscale, void* dw,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_norm(d)) return rc;
  if (!scale || !w || !dscale || !dw || (d->rows && (!o || !r || !d_o || !dr)))
    return fail(FESC_ERR_ARG, "null buffer");
  NormArgs n = norm_args(d, false, o, r, nullptr, scale, w);
  n.du = du;
  n.dr_new = dr_new;
  n.da = d_o;
  n.db = dr;
  n.dk = dscale;
  n.dw = dw;
  return norm_bwd(d, false, n, workspace, workspace_bytes, stream);
}

}  // extern "C"
