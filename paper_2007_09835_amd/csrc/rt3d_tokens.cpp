// Host side of librt3d's token operators: argument validation, launch rules and
// the C entry points declared in include/rt3d.h.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <numeric>

#include "rt3d_tokens.h"

namespace rt3d {
namespace {

constexpr int64_t kMaxRows = (1ll << 31) - 16;
constexpr int kMaxNormColumns = 1 << 20;
constexpr int64_t kMaxPitch = 1 << 22;   // elements: a tile's rows stay within 2^31 bytes
constexpr int kMaxLength = 1 << 30;
constexpr int kSplitBlocks = 2048;   // workgroups of one wave that a call of few queries is split into
constexpr int kSplitKeys = 256;      // least keys of such a split

bool known_dtype(int dtype) { return dtype == RT3D_F32 || dtype == RT3D_BF16 || dtype == RT3D_F16; }
int esize(int dtype) { return dtype == RT3D_F32 ? 4 : 2; }
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// A launch has fewer than 2^32 threads along its grid: HIP takes no more.
rt3d_status check_launch(int64_t workgroups, int threads, const char *what) {
  if (workgroups >= ((1ll << 32) + threads - 1) / threads)
    return fail(RT3D_ERR_UNSUPPORTED, "too many %s for one call: a launch of 2^32 threads", what);
  return RT3D_OK;
}

rt3d_status launched(int e) {
  if (e != hipSuccess)
    return fail(RT3D_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(static_cast<hipError_t>(e)));
  return ok();
}

// ---------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------

rt3d_status check_norm(const rt3d_norm_desc *d) {
  if (!d) return fail(RT3D_ERR_INVALID_ARG, "desc is NULL");
  if (d->rows < 0) return fail(RT3D_ERR_INVALID_ARG, "rows must be non-negative");
  if (d->c <= 0) return fail(RT3D_ERR_INVALID_ARG, "c must be positive");
  if (!known_dtype(d->dtype)) return fail(RT3D_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (!(d->eps > 0.f) || !std::isfinite(d->eps))
    return fail(RT3D_ERR_INVALID_ARG, "eps must be finite and > 0");
  if ((d->x_pitch && d->x_pitch < d->c) || (d->y_pitch && d->y_pitch < d->c))
    return fail(RT3D_ERR_INVALID_ARG, "pitches must be 0 or at least c");
  if (d->c > kMaxNormColumns) return fail(RT3D_ERR_UNSUPPORTED, "rows of more than %d channels", kMaxNormColumns);
  if (static_cast<double>(d->rows) * static_cast<double>(std::max({d->x_pitch, d->y_pitch, static_cast<int64_t>(d->c)})) >
      9.0e18 / 4)
    return fail(RT3D_ERR_UNSUPPORTED, "rows times pitch passes 64 bits");
  return RT3D_OK;
}

NormArgs norm_args(const rt3d_norm_desc *d) {
  NormArgs a{};
  a.rows = d->rows;
  a.c = d->c;
  a.eps = d->eps;
  a.x_pitch = d->x_pitch ? d->x_pitch : d->c;
  a.y_pitch = d->y_pitch ? d->y_pitch : d->c;
  a.blocks = layernorm_bwd_blocks(d->rows);
  return a;
}

uint64_t norm_workspace(const rt3d_norm_desc *d) {
  return static_cast<uint64_t>(layernorm_bwd_blocks(d->rows)) * 2 * d->c * sizeof(float);
}

// ---------------------------------------------------------------------------
// Rotation by positions
// ---------------------------------------------------------------------------

rt3d_status check_rope(const rt3d_rope_desc *d) {
  if (!d) return fail(RT3D_ERR_INVALID_ARG, "desc is NULL");
  if (d->n < 0 || d->t < 0) return fail(RT3D_ERR_INVALID_ARG, "n and t must be non-negative");
  if (d->h <= 0 || d->w <= 0 || d->vecs <= 0) return fail(RT3D_ERR_INVALID_ARG, "h, w and vecs must be positive");
  if (d->d <= 0 || d->d % 2) return fail(RT3D_ERR_INVALID_ARG, "d must be positive and even");
  if (d->dt < 0 || d->dh < 0 || d->dw < 0 || d->dt % 2 || d->dh % 2 || d->dw % 2)
    return fail(RT3D_ERR_INVALID_ARG, "sections must be non-negative and even");
  if (static_cast<int64_t>(d->dt) + d->dh + d->dw > d->d)
    return fail(RT3D_ERR_INVALID_ARG, "sections pass the vector's %d channels", d->d);
  if (!known_dtype(d->dtype)) return fail(RT3D_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (d->flags & ~(RT3D_ROPE_HALVES | RT3D_ROPE_INVERSE)) return fail(RT3D_ERR_INVALID_ARG, "unknown flags");
  if (!(d->base > 0.0) || !std::isfinite(d->base)) return fail(RT3D_ERR_INVALID_ARG, "base must be finite and > 0");
  if (d->t0 < 0 || static_cast<int64_t>(d->t0) + d->t > 0x7fffffffll)
    return fail(RT3D_ERR_INVALID_ARG, "positions t0 .. t0 + t must lie in 0 .. 2^31 - 1");
  const int64_t row = static_cast<int64_t>(d->vecs) * d->d;
  for (const rt3d_rows *r : {&d->x, &d->y}) {
    if (r->pitch && r->pitch < row) return fail(RT3D_ERR_INVALID_ARG, "pitches must be 0 or at least vecs * d");
    if (r->batch < 0) return fail(RT3D_ERR_INVALID_ARG, "batch strides must be non-negative");
  }
  if (static_cast<double>(d->h) * d->w * std::max(d->t, 1) > 2.0e9)
    return fail(RT3D_ERR_UNSUPPORTED, "more than 2e9 tokens in a clip");
  return RT3D_OK;
}

// ---------------------------------------------------------------------------
// Differential attention
// ---------------------------------------------------------------------------

struct Shape {
  int64_t q_row, k_row;  // elements of a token's queries (and outputs), keys (and values)
  int group;
};

rt3d_status check_rows(const rt3d_rows &r, int64_t row, int64_t len, int es, bool out, const char *what) {
  if (r.pitch && r.pitch < row) return fail(RT3D_ERR_INVALID_ARG, "%s: pitch below %lld", what, static_cast<long long>(row));
  if (r.batch < 0) return fail(RT3D_ERR_INVALID_ARG, "%s: batch stride is negative", what);
  const int64_t pitch = r.pitch ? r.pitch : row;
  if (out && r.batch && r.batch < (std::max<int64_t>(len, 1) - 1) * pitch + row)
    return fail(RT3D_ERR_INVALID_ARG, "%s: clips overlap", what);
  if (pitch >= kMaxPitch) return fail(RT3D_ERR_UNSUPPORTED, "%s: a token pitch of 2^22 elements or more", what);
  if (pitch * es % 16 || r.batch * es % 16)
    return fail(RT3D_ERR_UNSUPPORTED, "%s: strides must be multiples of 16 bytes", what);
  return RT3D_OK;
}

rt3d_status check_attn(const rt3d_diffattn_desc *d, bool backward, Shape &s) {
  if (!d) return fail(RT3D_ERR_INVALID_ARG, "desc is NULL");
  if (d->n < 0 || d->lq < 0 || d->lk < 0) return fail(RT3D_ERR_INVALID_ARG, "n, lq and lk must be non-negative");
  if (d->hq <= 0 || d->hk <= 0 || d->hq % d->hk)
    return fail(RT3D_ERR_INVALID_ARG, "hq must be a positive multiple of hk");
  if (d->d <= 0) return fail(RT3D_ERR_INVALID_ARG, "d must be positive");
  if (!known_dtype(d->dtype)) return fail(RT3D_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (d->frame < 0) return fail(RT3D_ERR_INVALID_ARG, "frame must be non-negative");
  if (!(d->scale >= 0.f) || !std::isfinite(d->scale))
    return fail(RT3D_ERR_INVALID_ARG, "scale must be finite and >= 0");
  if (d->d % 8 || d->d > 128) return fail(RT3D_ERR_UNSUPPORTED, "d must be a multiple of 8 up to 128, got %d", d->d);
  s.group = d->hq / d->hk;
  if (d->lq >= kMaxLength || d->lk >= kMaxLength || d->frame >= kMaxLength ||
      static_cast<int64_t>(d->lq) * s.group >= kMaxLength)
    return fail(RT3D_ERR_UNSUPPORTED, "lengths (times hq / hk) must be below 2^30");
  const double rows = static_cast<double>(d->n) * d->hk * (static_cast<double>(d->lq) * s.group + d->lk + 64);
  if (rows >= static_cast<double>(kMaxRows)) return fail(RT3D_ERR_UNSUPPORTED, "more than 2^31 rows");
  s.q_row = 2ll * d->hq * d->d;
  s.k_row = 2ll * d->hk * d->d;
  const int es = esize(d->dtype);
  rt3d_status st = RT3D_OK;
  auto rows_of = [&](const rt3d_rows &r, int64_t row, int len, bool out, const char *what) {
    if (st == RT3D_OK) st = check_rows(r, row, len, es, out, what);
  };
  rows_of(d->q, s.q_row, d->lq, false, "q");
  rows_of(d->k, s.k_row, d->lk, false, "k");
  rows_of(d->v, s.k_row, d->lk, false, "v");
  rows_of(d->o, s.q_row, d->lq, true, "o");
  if (backward) {
    rows_of(d->d_o, s.q_row, d->lq, false, "d_o");
    rows_of(d->dq, s.q_row, d->lq, true, "dq");
    rows_of(d->dk, s.k_row, d->lk, true, "dk");
    rows_of(d->dv, s.k_row, d->lk, true, "dv");
  }
  return st;
}

void put_rows(const rt3d_rows &r, int64_t row, int64_t len, int64_t &pitch, int64_t &batch) {
  pitch = r.pitch ? r.pitch : row;
  batch = r.batch ? r.batch : len * pitch;
}

AttnArgs attn_args(const rt3d_diffattn_desc *d, const Shape &s, bool lengths) {
  AttnArgs a{};
  // Clips of unlike lengths would leave XCDs idle while others work: 8 x 6272
  // tokens, 8 heads, d 64, forward 1623 us with a clip's head on one XCD, 937 over
  // all; 4 to 64 clips with 2 to 8 key heads 1.02-1.7x. The lengths are on the device,
  // so a call that is given any counts as unlike: clips that are in truth equal keep
  // the shared L2 only where no lengths are given.
  a.spread = lengths ? 1 : 0;
  if (d->frame) a.sets = lengths ? 1 : static_cast<int32_t>(std::gcd<int64_t>(static_cast<int64_t>(d->n) * d->hk, 8));
  a.n = d->n;
  a.lq = d->lq;
  a.lk = d->lk;
  a.hq = d->hq;
  a.hk = d->hk;
  a.d = d->d;
  a.group = s.group;
  a.frame = d->frame;
  a.scale = d->scale > 0.f ? d->scale : 1.f / std::sqrt(static_cast<float>(d->d));
  a.scale2 = a.scale * 1.44269504088896340736f;
  put_rows(d->q, s.q_row, d->lq, a.q_pitch, a.q_batch);
  put_rows(d->k, s.k_row, d->lk, a.k_pitch, a.k_batch);
  put_rows(d->v, s.k_row, d->lk, a.v_pitch, a.v_batch);
  put_rows(d->o, s.q_row, d->lq, a.o_pitch, a.o_batch);
  put_rows(d->d_o, s.q_row, d->lq, a.do_pitch, a.do_batch);
  put_rows(d->dq, s.q_row, d->lq, a.dq_pitch, a.dq_batch);
  put_rows(d->dk, s.k_row, d->lk, a.dk_pitch, a.dk_batch);
  put_rows(d->dv, s.k_row, d->lk, a.dv_pitch, a.dv_batch);
  return a;
}

// How many parts a workgroup's walk is split into.  blocks: workgroups of a call
// without splits, each a walk of `steps` steps of `step_us` on a CU of its own;
// part_bytes: one split's partial results, written and read once at 4 TB/s; a
// split call pays 5 us for its second launch.  The time is that of the fullest
// CU; workgroups that share one take `shared` of the sum of their times (16-bit
// ones fill each other's waits, 32-bit ones wait for the same matrix units).
// Two clips of 392 tokens in 32 bits: 7 splits of dq and dk/dv 31 and 36 us, 4
// splits 26 and 31, none 56 and 70.
// A causal call without splits takes as long as its longest walk, and its CUs share
// less, as most walks are shorter.  (Causal, forward and backward, without splits and
// with: 8000 tokens, 4 heads, d 64 649 and 494 us; 6000 tokens, 8 heads 736 and 559;
// 5 clips of 3000 tokens, 4 heads 410 and 409, the forward alone 99 and 100.)
constexpr int kCus = 256;

// Mean length of the walks of a causal call, as a share of the longest.
double walk_share(const rt3d_diffattn_desc *d) {
  if (!d->frame || d->frame >= d->lk) return 1.0;
  return d->lq <= d->lk ? 1.0 - 0.5 * d->lq / d->lk : 0.5 * d->lk / d->lq;
}
// `part(s)`: the steps of a walk that is asked for s splits, and how many that makes.
// At most `most` splits are made (and asked for at most `tries`).
template <typename Part>
int pick_splits(const rt3d_diffattn_desc *d, int64_t blocks, int64_t steps, double step_us, double part_bytes,
                int64_t tries, int64_t most, Part &&part) {
  const double share = walk_share(d);
  if (blocks <= 0 || blocks * share >= 2 * kCus || steps < 2) return 1;
  const double shared = d->dtype == RT3D_F32 ? 1.0 : 0.6;
  auto time = [&](int64_t walk, int64_t s) {
    const double on_cu = share * static_cast<double>((blocks * s + kCus - 1) / kCus);
    return walk * step_us * std::max(1.0, shared * on_cu) + (s > 1 ? 5.0 + 2 * s * part_bytes / 4e6 : 0.0);
  };
  int best = 1;
  double least = time(steps, 1);
  for (int64_t s = 2; s <= tries && s <= steps; ++s) {
    const auto [walk, made] = part(s);
    if (made < 2 || made > most) continue;
    const double t = time(walk, made);
    if (t < least) least = t, best = static_cast<int>(made);
  }
  return best;
}

// Keys of a split: whole staged tiles (of 32 or 64 keys), so that none reaches into
// the next.  That makes split_count splits, often fewer than asked for; asked for so
// many, the span is the same.  Plans are made of these counts, so that the workspace of
// one pays for it again.
int split_span(int lk, int64_t splits) { return static_cast<int>((lk + splits - 1) / splits + 63) / 64 * 64; }
int split_count(int lk, int span) { return static_cast<int>((static_cast<int64_t>(lk) + span - 1) / span); }

struct Walk {
  int64_t steps, splits;
};
int pick_key_splits(const rt3d_diffattn_desc *d, int64_t blocks, double step_us, double part_bytes, int64_t tries,
                    int64_t most) {
  return pick_splits(d, blocks, (d->lk + 31) / 32, step_us, part_bytes, tries, most, [&](int64_t s) {
    const int span = split_span(d->lk, s);
    return Walk{span / 32, split_count(d->lk, span)};
  });
}

// Time of a step of 32 keys (forward, dq) or 32 queries (dk, dv) of a workgroup
// alone on its CU, in us per 32 channels of d: 32-bit steps take their products
// (6144 or 8192 cycles of the matrix unit), 16-bit ones the rest as well.
double step_us(const rt3d_diffattn_desc *d, double bits16, double bits32) {
  const int wide = d->d <= 32 ? 1 : d->d <= 64 ? 2 : 4;
  return wide * (d->dtype == RT3D_F32 ? bits32 : bits16);
}

// Launch of a forward call: groups of 32 rows of a workgroup and splits of the keys.
struct FwdPlan {
  int row_groups, tiles, splits, span;
  int64_t blocks;
  uint64_t bytes;  // workspace
};

FwdPlan fwd_plan(const rt3d_diffattn_desc *d, const Shape &s, uint64_t workspace) {
  FwdPlan p{};
  const int64_t rows = static_cast<int64_t>(d->lq) * s.group, pairs = static_cast<int64_t>(d->n) * d->hk;
  // One group where more would leave waves without rows: then a workgroup is one
  // wave (two beyond d = 64) and a CU holds several.
  p.row_groups = rows <= 32 ? 1 : attn_row_groups(d->d);
  p.tiles = static_cast<int>((rows + 32 * p.row_groups - 1) / (32 * p.row_groups));
  p.blocks = pairs * p.tiles;
  p.splits = 1;
  p.span = d->lk;
  const uint64_t one = static_cast<uint64_t>(pairs * rows) * (4 + 4 * d->d) * sizeof(float);
  if (p.blocks <= 0) return p;
  constexpr int64_t kMost = 256;
  const int64_t most = std::min<int64_t>(kMost, static_cast<int64_t>(workspace / one));
  int64_t splits;
  if (p.row_groups == 1) {
    // bound by the cache's bytes: enough waves to keep them coming
    splits = std::min<int64_t>({most, kSplitBlocks / p.blocks, d->lk / kSplitKeys});
  } else {
    splits = pick_key_splits(d, p.blocks, step_us(d, 0.35, 2.9), static_cast<double>(one), kMost, most);
  }
  if (splits > 1) {
    p.span = split_span(d->lk, splits);
    p.splits = split_count(d->lk, p.span);
  }
  if (p.splits > 1) {
    p.blocks *= p.splits;
    p.bytes = one * p.splits;
  }
  return p;
}

BwdPlan bwd_plan(const rt3d_diffattn_desc *d, const Shape &s) {
  BwdPlan p{};
  const int64_t rows = static_cast<int64_t>(d->lq) * s.group, pairs = static_cast<int64_t>(d->n) * d->hk;
  const uint64_t stats = static_cast<uint64_t>(d->n) * d->hq * d->lq;
  const uint64_t dq = stats * 2 * d->d, dkv = static_cast<uint64_t>(pairs) * d->lk * 4 * d->d;
  p.dq_span = d->lk;
  p.dq_splits = pick_key_splits(d, pairs * ((rows + kBwdRows - 1) / kBwdRows), step_us(d, 0.35, 2.9), dq * 4.0, 16, 16);
  if (p.dq_splits > 1) p.dq_span = split_span(d->lk, p.dq_splits);
  const int64_t tiles = static_cast<int64_t>(s.group) * ((d->lq + 31) / 32);
  p.dkv_splits = pick_splits(d, pairs * ((d->lk + kBwdRows - 1) / kBwdRows), tiles, step_us(d, 0.45, 3.9), dkv * 4.0,
                             16, 16, [&](int64_t s) { return Walk{(tiles + s - 1) / s, s}; });
  auto up = [](uint64_t floats) { return (floats + 3) / 4 * 4; };  // parts begin at 16 bytes
  p.dq_part = up((2 + p.dq_splits) * stats);
  p.dkv_part = p.dq_part + (p.dq_splits > 1 ? up(p.dq_splits * dq) : 0);
  p.floats = p.dkv_part + (p.dkv_splits > 1 ? p.dkv_splits * dkv : 0);
  return p;
}

// Whether every launch of a call can be made (workgroups go round eight XCDs).
int64_t by_eight(int64_t workgroups) { return (workgroups + 7) / 8 * 8; }

rt3d_status check_fwd_launches(const rt3d_diffattn_desc *d, const FwdPlan &p) {
  rt3d_status st = check_launch(by_eight(p.blocks), attn_fwd_threads(d->d, p.row_groups), "rows");
  if (st == RT3D_OK && p.splits > 1) st = check_launch(static_cast<int64_t>(d->n) * d->hq * d->lq, 256, "rows");
  return st;
}

rt3d_status check_bwd_launches(const rt3d_diffattn_desc *d, const Shape &s, const BwdPlan &p) {
  const int64_t rows = static_cast<int64_t>(d->lq) * s.group, pairs = static_cast<int64_t>(d->n) * d->hk;
  auto tiles = [](int64_t len) { return (len + kBwdRows - 1) / kBwdRows; };
  rt3d_status st = check_launch(by_eight(pairs * tiles(rows) * p.dq_splits), kBwdThreads, "queries");
  if (st == RT3D_OK) st = check_launch(by_eight(pairs * tiles(d->lk) * p.dkv_splits) + d->hq, kBwdThreads, "keys");
  // the sums of the splits' gradients
  if (st == RT3D_OK && p.dq_splits > 1) st = check_launch((pairs * rows * d->d / 2 + 255) / 256, 256, "queries");
  if (st == RT3D_OK && p.dkv_splits > 1) st = check_launch((pairs * d->lk * d->d + 255) / 256, 256, "keys");
  return st;
}

}  // namespace
}  // namespace rt3d

using namespace rt3d;

extern "C" {

rt3d_status rt3d_layernorm_fwd(const rt3d_norm_desc *d, const void *x, const float *gamma, const float *beta,
                               void *y, float *mean, float *rstd, void *stream) {
  const rt3d_status st = check_norm(d);
  if (st != RT3D_OK) return st;
  if (d->rows == 0) return ok();
  if (!x || !y) return fail(RT3D_ERR_INVALID_ARG, "x and y must be non-NULL");
  const int es = esize(d->dtype);
  if (!aligned(x, es) || !aligned(y, es) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4))
    return fail(RT3D_ERR_INVALID_ARG, "pointers must be aligned to their element size");
  NormArgs a = norm_args(d);
  if (x == y && a.x_pitch != a.y_pitch)
    return fail(RT3D_ERR_INVALID_ARG, "a layer norm in place needs one pitch");
  a.x = x;
  a.y = y;
  a.gamma = gamma;
  a.beta = beta;
  a.mean = mean;
  a.rstd = rstd;
  return launched(launch_layernorm_fwd(a, d->dtype, stream));
}

rt3d_status rt3d_layernorm_bwd_workspace_size(const rt3d_norm_desc *d, uint64_t *bytes) {
  const rt3d_status st = check_norm(d);
  if (st != RT3D_OK) return st;
  if (!bytes) return fail(RT3D_ERR_INVALID_ARG, "bytes must be non-NULL");
  *bytes = norm_workspace(d);
  return ok();
}

rt3d_status rt3d_layernorm_bwd(const rt3d_norm_desc *d, const void *x, const void *dy, const float *gamma,
                               const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta,
                               void *workspace, uint64_t workspace_bytes, void *stream) {
  const rt3d_status st = check_norm(d);
  if (st != RT3D_OK) return st;
  const bool weights = dgamma || dbeta;
  if (!dx && !weights) return ok();
  if (d->rows > 0 && (!x || !dy || !mean || !rstd))
    return fail(RT3D_ERR_INVALID_ARG, "x, dy, mean and rstd must be non-NULL");
  const int es = esize(d->dtype);
  if (!aligned(x, es) || !aligned(dy, es) || !aligned(dx, es) || !aligned(gamma, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4) || !aligned(workspace, 4))
    return fail(RT3D_ERR_INVALID_ARG, "pointers must be aligned to their element size");
  if (weights && (!workspace || workspace_bytes < norm_workspace(d)))
    return fail(RT3D_ERR_BUFFER_TOO_SMALL, "dgamma and dbeta need %llu bytes of workspace, got %llu",
                static_cast<unsigned long long>(norm_workspace(d)),
                static_cast<unsigned long long>(workspace ? workspace_bytes : 0));
  if (d->rows == 0 && !weights) return ok();
  NormArgs a = norm_args(d);
  a.x = x;
  a.dy = dy;
  a.gamma = gamma;
  a.mean = const_cast<float *>(mean);
  a.rstd = const_cast<float *>(rstd);
  a.dx = dx;
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.partial = weights ? static_cast<float *>(workspace) : nullptr;
  return launched(launch_layernorm_bwd(a, d->dtype, stream));
}

rt3d_status rt3d_rope3d(const rt3d_rope_desc *d, const void *x, const int32_t *pos, void *y, void *stream) {
  const rt3d_status st = check_rope(d);
  if (st != RT3D_OK) return st;
  RopeArgs a{};
  a.tokens = static_cast<int64_t>(d->t) * d->h * d->w;
  if (d->n == 0 || a.tokens == 0) return ok();
  if (!x || !y) return fail(RT3D_ERR_INVALID_ARG, "x and y must be non-NULL");
  const int es = esize(d->dtype);
  if (!aligned(x, es) || !aligned(y, es) || !aligned(pos, 4))
    return fail(RT3D_ERR_INVALID_ARG, "pointers must be aligned to their element size");
  a.x = x;
  a.y = y;
  a.pos = pos;
  put_rows(d->x, static_cast<int64_t>(d->vecs) * d->d, a.tokens, a.x_pitch, a.x_batch);
  put_rows(d->y, static_cast<int64_t>(d->vecs) * d->d, a.tokens, a.y_pitch, a.y_batch);
  if (d->n > 1 && a.y_batch < (a.tokens - 1) * a.y_pitch + static_cast<int64_t>(d->vecs) * d->d)
    return fail(RT3D_ERR_INVALID_ARG, "clips of y overlap");
  if (x == y && (a.x_pitch != a.y_pitch || a.x_batch != a.y_batch))
    return fail(RT3D_ERR_INVALID_ARG, "a rotation in place needs one layout");
  a.base_log2 = std::log2(d->base);
  a.n = d->n;
  a.h = d->h;
  a.w = d->w;
  a.vecs = d->vecs;
  a.d = d->d;
  a.size[0] = d->dt;
  a.size[1] = d->dh;
  a.size[2] = d->dw;
  a.t0 = d->t0;
  a.inverse = d->flags & RT3D_ROPE_INVERSE ? 1 : 0;
  const int halves = d->flags & RT3D_ROPE_HALVES ? 1 : 0;
  // The widest access (16 bytes at most) whose runs end with the vector (and the sections' halves).
  int pairs = halves ? 16 / es : 8 / es;
  const int rest = d->d - d->dt - d->dh - d->dw;
  auto fits = [&](int p) {
    if (!halves) return d->d % (2 * p) == 0;
    return d->dt / 2 % p == 0 && d->dh / 2 % p == 0 && d->dw / 2 % p == 0 && rest / 2 % p == 0;
  };
  while (!fits(pairs)) pairs /= 2;  // one pair always fits: d and the sections are even
  a.slots = d->d / 2 / pairs;
  const int64_t base = static_cast<int64_t>(d->n) * a.tokens * a.slots;
  constexpr int64_t kThreads = 512 * 1024;  // two waves of threads for every SIMD's eight
  a.chunks = static_cast<int>(std::min<int64_t>(d->vecs, std::max<int64_t>(1, (kThreads + base - 1) / base)));
  a.threads = base * a.chunks;
  const rt3d_status can = check_launch((a.threads + 255) / 256, 256, "vectors");
  if (can != RT3D_OK) return can;
  return launched(launch_rope(a, d->dtype, halves, pairs, stream));
}

rt3d_status rt3d_diffattn_fwd_workspace_size(const rt3d_diffattn_desc *d, uint64_t *bytes) {
  Shape s;
  const rt3d_status st = check_attn(d, false, s);
  if (st != RT3D_OK) return st;
  if (!bytes) return fail(RT3D_ERR_INVALID_ARG, "bytes must be non-NULL");
  const FwdPlan p = fwd_plan(d, s, ~0ull);
  const rt3d_status fits = check_fwd_launches(d, p);
  if (fits != RT3D_OK) return fits;
  *bytes = p.bytes;
  return ok();
}

rt3d_status rt3d_diffattn_fwd(const rt3d_diffattn_desc *d, const void *q, const void *k, const void *v,
                              const float *lambda, const int32_t *q_len, const int32_t *k_len, void *o, void *o2,
                              float *lse, void *workspace, uint64_t workspace_bytes, void *stream) {
  Shape s;
  const rt3d_status st = check_attn(d, false, s);
  if (st != RT3D_OK) return st;
  if (d->n == 0 || d->lq == 0) return ok();
  if (!q || !lambda || !o || (d->lk > 0 && (!k || !v)))
    return fail(RT3D_ERR_INVALID_ARG, "q, k, v, lambda and o must be non-NULL");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(o2, 16) ||
      !aligned(workspace, 16))
    return fail(RT3D_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
  if (!aligned(lambda, 4) || !aligned(lse, 4) || !aligned(q_len, 4) || !aligned(k_len, 4))
    return fail(RT3D_ERR_INVALID_ARG, "lambda, lse and lengths must be 4-byte aligned");
  const FwdPlan p = fwd_plan(d, s, workspace ? workspace_bytes : 0);
  const rt3d_status fits = check_fwd_launches(d, p);
  if (fits != RT3D_OK) return fits;
  AttnArgs a = attn_args(d, s, q_len || k_len);
  a.q = q;
  a.k = k;
  a.v = v;
  a.lam = lambda;
  a.q_len = q_len;
  a.k_len = k_len;
  a.out = o;
  a.out2 = o2;
  a.lse = lse;
  a.part = static_cast<float *>(workspace);
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.span = p.span;
  a.blocks = p.blocks;
  return launched(launch_attn_fwd(a, d->dtype, p.row_groups, stream));
}

rt3d_status rt3d_diffattn_bwd_workspace_size(const rt3d_diffattn_desc *d, uint64_t *bytes) {
  Shape s;
  const rt3d_status st = check_attn(d, true, s);
  if (st != RT3D_OK) return st;
  if (!bytes) return fail(RT3D_ERR_INVALID_ARG, "bytes must be non-NULL");
  const BwdPlan p = bwd_plan(d, s);
  const rt3d_status fits = check_bwd_launches(d, s, p);
  if (fits != RT3D_OK) return fits;
  *bytes = p.floats * sizeof(float);
  return ok();
}

rt3d_status rt3d_diffattn_bwd(const rt3d_diffattn_desc *d, const void *q, const void *k, const void *v,
                              const float *lambda, const int32_t *q_len, const int32_t *k_len, const void *o,
                              const void *o2, const float *lse, const void *d_o, void *dq, void *dk, void *dv,
                              float *dlambda, void *workspace, uint64_t workspace_bytes, void *stream) {
  Shape s;
  const rt3d_status st = check_attn(d, true, s);
  if (st != RT3D_OK) return st;
  if (!dq && !dk && !dv && !dlambda) return ok();
  const bool queries = d->n > 0 && d->lq > 0, keys = d->n > 0 && d->lk > 0;
  if (queries && (!q || !lambda || !o || !o2 || !lse || !d_o))
    return fail(RT3D_ERR_INVALID_ARG, "q, lambda, o, o2, lse and d_o must be non-NULL");
  if (keys && (!k || !v)) return fail(RT3D_ERR_INVALID_ARG, "k and v must be non-NULL");
  for (const void *x : {q, k, v, o, o2, d_o, static_cast<const void *>(dq), static_cast<const void *>(dk),
                        static_cast<const void *>(dv), static_cast<const void *>(workspace)})
    if (!aligned(x, 16)) return fail(RT3D_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
  if (!aligned(lambda, 4) || !aligned(lse, 4) || !aligned(dlambda, 4) || !aligned(q_len, 4) || !aligned(k_len, 4))
    return fail(RT3D_ERR_INVALID_ARG, "lambda, dlambda, lse and lengths must be 4-byte aligned");
  const BwdPlan p = bwd_plan(d, s);
  const rt3d_status fits = check_bwd_launches(d, s, p);
  if (fits != RT3D_OK) return fits;
  const uint64_t need = p.floats * sizeof(float);
  if (need && (!workspace || workspace_bytes < need))
    return fail(RT3D_ERR_BUFFER_TOO_SMALL, "the backward pass needs %llu bytes of workspace, got %llu",
                static_cast<unsigned long long>(need),
                static_cast<unsigned long long>(workspace ? workspace_bytes : 0));
  AttnArgs a = attn_args(d, s, q_len || k_len);
  a.q = q;
  a.k = k;
  a.v = v;
  a.lam = lambda;
  a.q_len = q_len;
  a.k_len = k_len;
  a.o = o;
  a.o2 = o2;
  a.lse = const_cast<float *>(lse);
  a.d_o = d_o;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dlam = dlambda;
  a.rowstat = static_cast<float *>(workspace);
  return launched(launch_attn_bwd(a, p, d->dtype, stream));
}

}  // extern "C"
