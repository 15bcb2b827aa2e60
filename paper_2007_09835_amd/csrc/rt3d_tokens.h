// Internal definitions of the token operators (layer norm, rotary positions,
// differential attention), shared by their host side and kernels.  Not part of
// the public ABI.
#pragma once

#include <stdint.h>

#include "../../include/rt3d.h"

namespace rt3d {

// The calling thread's error message (rt3d_host.cpp).
rt3d_status fail(rt3d_status s, const char *fmt, ...);
rt3d_status ok();

struct NormArgs {
  const void *x, *dy;
  void *y, *dx;               // the forward writes y, the backward dx
  const float *gamma, *beta;  // NULL: ones, zeros
  float *mean, *rstd;         // [rows]; the forward writes them (or NULL), the backward reads them
  float *dgamma, *dbeta;      // [c] or NULL
  float *partial;             // [blocks][2][c] sums of the backward's workgroups
  int64_t rows, x_pitch, y_pitch;
  int32_t c, blocks;
  float eps;
};

struct RopeArgs {
  const void *x;
  void *y;
  const int32_t *pos;  // [n][tokens][3], or NULL: the token's place in the grid
  int64_t x_pitch, x_batch, y_pitch, y_batch;
  int64_t tokens, threads;
  double base_log2;
  int32_t n, h, w, vecs, d;
  int32_t size[3];     // channels of the three sections
  int32_t t0;          // first frame's position (grid positions)
  int32_t slots, chunks;  // threads along a vector; vectors of a token are dealt to `chunks` threads
  int32_t inverse;
};

struct AttnArgs {
  const void *q, *k, *v, *o, *o2, *d_o;
  void *out, *out2;           // forward: o, and the second map's output (or NULL)
  void *dq, *dk, *dv;
  const float *lam;           // [hq]
  float *lse;                 // [2][n][hq][lq], base-2 logarithms (forward writes, or NULL)
  const int32_t *q_len, *k_len;
  float *part;                // partial results of split calls
  float *rowstat;             // backward: [2][n][hq][lq] row sums, then [dq splits][n][hq][lq] sums of P_2 dP
  float *dlam;                // [hq]
  int64_t q_pitch, k_pitch, v_pitch, o_pitch;
  int64_t q_batch, k_batch, v_batch, o_batch;
  int64_t do_pitch, dq_pitch, dk_pitch, dv_pitch;
  int64_t do_batch, dq_batch, dk_batch, dv_batch;
  int64_t blocks;             // workgroups that have work
  int32_t n, lq, lk, hq, hk, d, group, frame;
  int32_t tiles;              // row (or key) tiles of a (clip, key head)
  int32_t splits, span;       // splits of the other axis and its extent in a split
  int32_t stat_splits;        // splits of the dq kernel, whose sums of P_2 dP are added up
  int32_t dlam_blocks;        // workgroups of the dk/dv launch that do so (hq, or 0)
  int32_t spread;             // workgroups of a (clip, key head) go to all XCDs
  int32_t sets;               // causal: (clip, key head) pairs are this many sets, dealt to the XCDs; else 0
  float scale, scale2;        // scale2 = scale * log2(e)
};

// Launchers: hipSuccess or the launch error.
int launch_layernorm_fwd(const NormArgs &a, int dtype, void *stream);
int launch_layernorm_bwd(const NormArgs &a, int dtype, void *stream);
// Workgroups of the backward pass, which is the count of its partial sums.
int layernorm_bwd_blocks(int64_t rows);

int launch_rope(const RopeArgs &a, int dtype, int halves, int pairs, void *stream);

// Groups of 32 rows that a workgroup of a call without splits holds, 1 or this.
constexpr int attn_row_groups(int d) { return d > 64 ? 2 : 4; }
constexpr int attn_fwd_threads(int d, int row_groups) { return 64 * row_groups * (d > 64 ? 2 : 1); }
int launch_attn_fwd(const AttnArgs &a, int dtype, int row_groups, void *stream);

// Splits of the backward kernels' walks (keys for dq, query tiles for dk and dv),
// and where their partial results lie in the workspace (floats).
struct BwdPlan {
  int dq_splits, dq_span, dkv_splits;
  uint64_t dq_part, dkv_part, floats;
};
constexpr int kBwdRows = 128;  // rows (keys) of a backward workgroup, 32 a wave
constexpr int kBwdThreads = kBwdRows / 32 * 64;
int launch_attn_bwd(const AttnArgs &a, const BwdPlan &p, int dtype, void *stream);

}  // namespace rt3d
