// HIP kernels of librt3d for gfx950 (MI355X): layer norm (forward, backward with
// the gradients of its weights) and the rotation of vectors by their token's
// position along time, height and width.  All of them move every input and
// output once and are bound by memory.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "rt3d_tokens.h"

namespace rt3d {
namespace {

// V elements in one access of up to 16 bytes, at any element's address (global
// memory takes unaligned vectors; on this card they cost what their lines cost).
template <typename T, int V>
struct Pack {
  T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> get(const T *p) {
  Pack<T, V> x;
  __builtin_memcpy(&x, p, sizeof(x));
  return x;
}
template <typename T, int V>
__device__ __forceinline__ void put(T *p, const Pack<T, V> &x) {
  __builtin_memcpy(p, &x, sizeof(x));
}

// V elements of a row from column `col` on, as floats; columns from c on are zero
// and never read.
template <typename T, int V>
__device__ __forceinline__ void load_row(const T *p, int col, int c, float (&out)[V]) {
  if (col + V <= c) {
    const Pack<T, V> x = get<T, V>(p + col);
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = static_cast<float>(x.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = col + e < c ? static_cast<float>(p[col + e]) : 0.f;
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_row(T *p, int col, int c, const float (&in)[V]) {
  if (col + V <= c) {
    Pack<T, V> x;
#pragma unroll
    for (int e = 0; e < V; ++e) x.v[e] = static_cast<T>(in[e]);
    put(p + col, x);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (col + e < c) p[col + e] = static_cast<T>(in[e]);
  }
}

// A weight vector's elements; `none` where it is absent.
template <int V>
__device__ __forceinline__ void load_weight(const float *p, int col, int c, float none, float (&out)[V]) {
  if (p) {
    load_row(p, col, c, out);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = none;
  }
}

// The sum of a value over 2 S neighbouring lanes that hold equal sums over S.
template <int S>
__device__ __forceinline__ float lane_step(float v) {
  const unsigned u = __float_as_uint(v);
  if constexpr (S == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else if constexpr (S == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
    constexpr int kDpp = S == 1 ? 0xb1 : S == 2 ? 0x4e : S == 4 ? 0x141 : 0x140;
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(u), kDpp, 0xf, 0xf, true));
  }
}

// Sums of N values over the LPR lanes of a row (a power of two up to 64, or the
// whole workgroup of 256); every lane gets them.  The order is fixed; no step goes
// through LDS but the last one of a workgroup.
template <int LPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float *lds) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = lane_step<1>(v[i]);
    v[i] = lane_step<2>(v[i]);
    v[i] = lane_step<4>(v[i]);
    if constexpr (LPR >= 16) v[i] = lane_step<8>(v[i]);
    if constexpr (LPR >= 32) v[i] = lane_step<16>(v[i]);
    if constexpr (LPR >= 64) v[i] = lane_step<32>(v[i]);
  }
  if constexpr (LPR > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // the last sums have been read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (lds[i] + lds[N + i]) + (lds[2 * N + i] + lds[3 * N + i]);
  }
}

constexpr int kNormThreads = 256;

// A product that is rounded by itself, in no fma: every reader sees the same mean.
__device__ __forceinline__ float mean_of(float sum, float inv) {
#pragma clang fp contract(off)
  return sum * inv;
}

// Variance about a row's mean, from the sums of the distances to a first one and of
// their squares.  The first mean, of sums that round at the size of x, may lie a few
// steps off: much, where the row's spread is small (a constant row of 1000 in 32 bits:
// y = -0.02 with it).  off, the distances' own mean, is what it lacks.
__device__ __forceinline__ float variance(const float (&s)[2], float inv, float off) {
  const float v = fmaf(-off, off, s[1] * inv);  // (infinite, not NaN, where the squares are)
  return v < 0.f ? 0.f : v;
}

// Layer norm, rows in registers: LPR lanes hold a row, NV vectors of V elements
// each, so x is read once and the variance is the mean of squared distances (a
// second pass over registers, not a difference of sums of x).  A workgroup walks rows
// with its weights in registers.
template <typename T, int V, int NV, int LPR>
__global__ __launch_bounds__(kNormThreads) void layernorm_fwd_kernel(NormArgs a) {
  __shared__ float lds[8];
  constexpr int kRows = kNormThreads / LPR;
  const int lane = threadIdx.x % LPR;
  float g[NV][V], b[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    load_weight(a.gamma, (i * LPR + lane) * V, a.c, 1.f, g[i]);
    load_weight(a.beta, (i * LPR + lane) * V, a.c, 0.f, b[i]);
  }
  const float inv = 1.f / static_cast<float>(a.c);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.rows; base += step) {
    const int64_t row = base + threadIdx.x / LPR;
    const bool in = row < a.rows;
    const T *x = static_cast<const T *>(a.x) + (in ? row : 0) * a.x_pitch;
    float v[NV][V], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) load_row(x, (i * LPR + lane) * V, in ? a.c : 0, v[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += v[i][e];
    row_sum<LPR>(s, lds);
    const float mean = mean_of(s[0], inv);
    float far[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[i][e] = (i * LPR + lane) * V + e < a.c ? v[i][e] - mean : 0.f;
        far[0] += v[i][e];
        far[1] += v[i][e] * v[i][e];
      }
    row_sum<LPR>(far, lds);
    const float off = mean_of(far[0], inv), rstd = 1.f / sqrtf(variance(far, inv, off) + a.eps);
    if (!in) continue;
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean + off;
      if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_pitch;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = fmaf(fmaf(v[i][e], rstd, -off * rstd), g[i][e], b[i][e]);
      store_row(y, (i * LPR + lane) * V, a.c, v[i]);
    }
  }
}

// Rows too long for registers: a workgroup reads a row three times, the second and
// third time from cache.
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void layernorm_fwd_long_kernel(NormArgs a) {
  __shared__ float lds[8];
  const float inv = 1.f / static_cast<float>(a.c);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + row * a.x_pitch;
    T *y = static_cast<T *>(a.y) + row * a.y_pitch;
    float s[1] = {0.f}, v[V];
    for (int col = threadIdx.x * V; col < a.c; col += kNormThreads * V) {
      load_row(x, col, a.c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += v[e];
    }
    row_sum<256>(s, lds);
    const float mean = mean_of(s[0], inv);
    float far[2] = {0.f, 0.f};
    for (int col = threadIdx.x * V; col < a.c; col += kNormThreads * V) {
      load_row(x, col, a.c, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float w = col + e < a.c ? v[e] - mean : 0.f;
        far[0] += w;
        far[1] += w * w;
      }
    }
    row_sum<256>(far, lds);
    const float off = mean_of(far[0], inv), rstd = 1.f / sqrtf(variance(far, inv, off) + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean + off;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (int col = threadIdx.x * V; col < a.c; col += kNormThreads * V) {
      float g[V], b[V];
      load_row(x, col, a.c, v);
      load_weight(a.gamma, col, a.c, 1.f, g);
      load_weight(a.beta, col, a.c, 0.f, b);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = fmaf(fmaf(v[e] - mean, rstd, -off * rstd), g[e], b[e]);
      store_row(y, col, a.c, v);
    }
  }
}

// Backward: with h = (x - mean) rstd and w = dy gamma,
//   dx = rstd (w - mean_c(w) - h mean_c(w h)),  dgamma = sum_rows dy h,  dbeta = sum_rows dy.
// A workgroup walks rows, keeps its share of dgamma and dbeta in registers and
// leaves it, summed over its row groups in order, in partial[block].
template <typename T, int V, int NV, int LPR>
__global__ __launch_bounds__(kNormThreads) void layernorm_bwd_kernel(NormArgs a) {
  constexpr int kRows = kNormThreads / LPR;
  __shared__ float lds[kRows > 1 ? kRows * LPR * NV * V : 8];
  const int lane = threadIdx.x % LPR;
  float g[NV][V], dg[NV][V] = {}, db[NV][V] = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) load_weight(a.gamma, (i * LPR + lane) * V, a.c, 1.f, g[i]);
  const float inv = 1.f / static_cast<float>(a.c);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.rows; base += step) {
    const int64_t row = base + threadIdx.x / LPR;
    const bool in = row < a.rows;
    const int64_t r = in ? row : 0;
    const T *x = static_cast<const T *>(a.x) + r * a.x_pitch;
    const T *dy = static_cast<const T *>(a.dy) + r * a.y_pitch;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float h[NV][V], w[NV][V], s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      load_row(x, (i * LPR + lane) * V, in ? a.c : 0, h[i]);
      load_row(dy, (i * LPR + lane) * V, in ? a.c : 0, w[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        h[i][e] = (h[i][e] - mean) * rstd;  // columns past c: w is zero there
        dg[i][e] += w[i][e] * h[i][e];
        db[i][e] += w[i][e];
        w[i][e] *= g[i][e];
        s[0] += w[i][e];
        s[1] += w[i][e] * h[i][e];
      }
    row_sum<LPR>(s, lds);
    if (!in || !a.dx) continue;
    T *dx = static_cast<T *>(a.dx) + row * a.x_pitch;
    const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) w[i][e] = rstd * (w[i][e] - m0 - h[i][e] * m1);
      store_row(dx, (i * LPR + lane) * V, a.c, w[i]);
    }
  }
  if (!a.partial) return;
  float *out = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.c;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (kRows > 1) {
      constexpr int kCols = LPR * NV * V;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e)
          lds[(threadIdx.x / LPR) * kCols + (i * LPR + lane) * V + e] = k ? db[i][e] : dg[i][e];
      __syncthreads();
      for (int col = threadIdx.x; col < kCols && col < a.c; col += kNormThreads) {
        float s = 0.f;
#pragma unroll 4
        for (int r = 0; r < kRows; ++r) s += lds[r * kCols + col];
        out[k * a.c + col] = s;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int col = (i * LPR + lane) * V + e;
          if (col < a.c) out[k * a.c + col] = k ? db[i][e] : dg[i][e];
        }
    }
  }
}

// Rows too long for registers: dx as above in two reads, and the weights'
// gradients by columns, each workgroup over a run of rows.
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void layernorm_dx_long_kernel(NormArgs a) {
  __shared__ float lds[8];
  const float inv = 1.f / static_cast<float>(a.c);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + row * a.x_pitch;
    const T *dy = static_cast<const T *>(a.dy) + row * a.y_pitch;
    T *dx = static_cast<T *>(a.dx) + row * a.x_pitch;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f}, h[V], w[V], g[V];
    for (int col = threadIdx.x * V; col < a.c; col += kNormThreads * V) {
      load_row(x, col, a.c, h);
      load_row(dy, col, a.c, w);
      load_weight(a.gamma, col, a.c, 1.f, g);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[0] += w[e] * g[e];
        s[1] += w[e] * g[e] * ((h[e] - mean) * rstd);
      }
    }
    row_sum<256>(s, lds);
    const float m0 = s[0] * inv, m1 = s[1] * inv;
    for (int col = threadIdx.x * V; col < a.c; col += kNormThreads * V) {
      load_row(x, col, a.c, h);
      load_row(dy, col, a.c, w);
      load_weight(a.gamma, col, a.c, 1.f, g);
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = rstd * (w[e] * g[e] - m0 - (h[e] - mean) * rstd * m1);
      store_row(dx, col, a.c, w);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kNormThreads) void layernorm_columns_kernel(NormArgs a) {
  const int col = blockIdx.x * kNormThreads + threadIdx.x;
  if (col >= a.c) return;
  const int64_t per = (a.rows + a.blocks - 1) / a.blocks;
  const int64_t r0 = blockIdx.y * per, r1 = r0 + per < a.rows ? r0 + per : a.rows;
  float dg = 0.f, db = 0.f;
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    const float dy = static_cast<float>(static_cast<const T *>(a.dy)[r * a.y_pitch + col]);
    const float x = static_cast<float>(static_cast<const T *>(a.x)[r * a.x_pitch + col]);
    dg += dy * ((x - a.mean[r]) * a.rstd[r]);
    db += dy;
  }
  float *out = a.partial + static_cast<int64_t>(blockIdx.y) * 2 * a.c;
  out[col] = dg;
  out[a.c + col] = db;
}

// dgamma and dbeta: the workgroups' partial sums, kFinalRuns runs of them added in
// order by as many threads of a column, and then the runs.
constexpr int kFinalCols = 16, kFinalRuns = 64;
__global__ __launch_bounds__(kFinalCols * kFinalRuns) void layernorm_finalize_kernel(NormArgs a) {
  __shared__ float lds[kFinalRuns][kFinalCols];
  const int c2 = 2 * a.c;
  const int col = blockIdx.x * kFinalCols + threadIdx.x % kFinalCols, run = threadIdx.x / kFinalCols;
  float s = 0.f;
  if (col < c2) {
#pragma unroll 8
    for (int b = run; b < a.blocks; b += kFinalRuns) s += a.partial[static_cast<int64_t>(b) * c2 + col];
  }
  lds[run][threadIdx.x % kFinalCols] = s;
  __syncthreads();
  for (int w = kFinalRuns / 2; w > 0; w >>= 1) {
    if (run < w) lds[run][threadIdx.x % kFinalCols] += lds[run + w][threadIdx.x % kFinalCols];
    __syncthreads();
  }
  if (run || col >= c2) return;
  s = lds[0][threadIdx.x];
  if (col < a.c) {
    if (a.dgamma) a.dgamma[col] = s;
  } else if (a.dbeta) {
    a.dbeta[col - a.c] = s;
  }
}

// ---------------------------------------------------------------------------
// Rotation by positions
// ---------------------------------------------------------------------------

// Channels (first, second) of a pair turn by the angle pos * base^(-2 i / size)
// of pair i of their section.  A thread keeps the sines of its P pairs of one
// token and turns them in every vector that it is dealt.  Angles are formed and
// reduced to one turn in 64 bits (a position times a frequency loses its fraction
// of a turn in 32), sine and cosine of the rest are 32-bit.
//   HALVES = false: a pair is two neighbours, a thread has 2 P channels in a row;
//   HALVES = true: pair i of a section of s channels is (i, i + s/2); two runs of P.
// Channels behind the three sections are copied.
template <typename T, int P, bool HALVES>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (id >= a.threads) return;
  const int slot = static_cast<int>(id % a.slots);
  const int64_t rest = id / a.slots;
  const int chunk = static_cast<int>(rest % a.chunks);
  const int64_t tok = rest / a.chunks;  // over clips and their tokens
  const int64_t clip = tok / a.tokens, token = tok - clip * a.tokens;
  int pos[3];
  if (a.pos) {
#pragma unroll
    for (int i = 0; i < 3; ++i) pos[i] = a.pos[tok * 3 + i];
  } else {
    const int64_t hw = static_cast<int64_t>(a.h) * a.w;
    const int in = static_cast<int>(token % hw);
    pos[0] = static_cast<int>(token / hw) + a.t0;
    pos[1] = in / a.w;
    pos[2] = in % a.w;
  }
  float sn[P], cs[P];
  bool turn[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    int p = slot * P + j, axis = 0;
    if (2 * p >= a.size[0]) {
      p -= a.size[0] / 2;
      axis = 1;
      if (2 * p >= a.size[1]) {
        p -= a.size[1] / 2;
        axis = 2;
      }
    }
    const int size = a.size[axis];
    turn[j] = 2 * p < size;
    const double freq = turn[j] ? exp2(-2.0 * p / size * a.base_log2) : 0.0;
    double rev = static_cast<double>(pos[axis]) * freq * 0.15915494309189533577;
    rev -= rint(rev);
    sincospif(2.f * static_cast<float>(rev), &sn[j], &cs[j]);
    if (a.inverse) sn[j] = -sn[j];
  }
  // first channels of the thread's two runs
  int first = 2 * P * slot, second = first + 1;
  if constexpr (HALVES) {
    int p = slot * P, at = 0, size = a.size[0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (2 * p >= size) {
        p -= size / 2;
        at += size;
        size = i < 3 ? a.size[i] : a.d - at;
      }
    first = at + p;
    second = first + size / 2;
  }
  const T *x = static_cast<const T *>(a.x) + clip * a.x_batch + token * a.x_pitch;
  T *y = static_cast<T *>(a.y) + clip * a.y_batch + token * a.y_pitch;
#pragma unroll 4
  for (int v = chunk; v < a.vecs; v += a.chunks) {
    const T *xv = x + static_cast<int64_t>(v) * a.d;
    T *yv = y + static_cast<int64_t>(v) * a.d;
    T p0[P], p1[P];
    if constexpr (HALVES) {
      const Pack<T, P> u = get<T, P>(xv + first), w = get<T, P>(xv + second);
#pragma unroll
      for (int j = 0; j < P; ++j) p0[j] = u.v[j], p1[j] = w.v[j];
    } else {
      const Pack<T, 2 * P> u = get<T, 2 * P>(xv + first);
#pragma unroll
      for (int j = 0; j < P; ++j) p0[j] = u.v[2 * j], p1[j] = u.v[2 * j + 1];
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const float f = static_cast<float>(p0[j]), s = static_cast<float>(p1[j]);
      if (turn[j]) {
        p0[j] = static_cast<T>(f * cs[j] - s * sn[j]);
        p1[j] = static_cast<T>(f * sn[j] + s * cs[j]);
      }
    }
    if constexpr (HALVES) {
      Pack<T, P> u, w;
#pragma unroll
      for (int j = 0; j < P; ++j) u.v[j] = p0[j], w.v[j] = p1[j];
      put(yv + first, u);
      put(yv + second, w);
    } else {
      Pack<T, 2 * P> u;
#pragma unroll
      for (int j = 0; j < P; ++j) u.v[2 * j] = p0[j], u.v[2 * j + 1] = p1[j];
      put(yv + first, u);
    }
  }
}

// ---------------------------------------------------------------------------
// Launch rules
// ---------------------------------------------------------------------------

constexpr int kNormBlocks = 1024;  // four workgroups of four waves on each of 256 CUs

// Lanes of a row and vectors of a lane for c columns: the fewest lanes that hold
// the row in one vector each, then more vectors, then a whole workgroup.
// f(lanes, vectors) launches; false: the row is too long for registers.
template <int V, typename F>
bool pick_shape(int c, F &&f) {
  using std::integral_constant;
#define RT3D_SHAPE(L, N)                                                              \
  if (c <= (L) * (N) * V) {                                                           \
    f(integral_constant<int, (L)>{}, integral_constant<int, (N)>{});                  \
    return true;                                                                      \
  }
  RT3D_SHAPE(8, 1)
  RT3D_SHAPE(16, 1)
  RT3D_SHAPE(32, 1)
  RT3D_SHAPE(64, 1)
  RT3D_SHAPE(64, 2)
  RT3D_SHAPE(64, 4)
  RT3D_SHAPE(256, 2)
  RT3D_SHAPE(256, 4)
#undef RT3D_SHAPE
  return false;
}

template <typename T, int V>
void norm_fwd(const NormArgs &a, hipStream_t s) {
  const bool done = pick_shape<V>(a.c, [&](auto lanes, auto vectors) {
    constexpr int L = decltype(lanes)::value, N = decltype(vectors)::value;
    const int64_t want = (a.rows + 256 / L - 1) / (256 / L);
    layernorm_fwd_kernel<T, V, N, L>
        <<<static_cast<unsigned>(std::min<int64_t>(want, 2 * kNormBlocks)), kNormThreads, 0, s>>>(a);
  });
  if (!done)
    layernorm_fwd_long_kernel<T, V>
        <<<static_cast<unsigned>(std::min<int64_t>(a.rows, 2 * kNormBlocks)), kNormThreads, 0, s>>>(a);
}

template <typename T, int V>
void norm_bwd(const NormArgs &a, hipStream_t s) {
  const bool done = pick_shape<V>(a.c, [&](auto lanes, auto vectors) {
    constexpr int L = decltype(lanes)::value, N = decltype(vectors)::value;
    layernorm_bwd_kernel<T, V, N, L><<<a.blocks, kNormThreads, 0, s>>>(a);
  });
  if (!done) {
    if (a.dx && a.rows > 0)
      layernorm_dx_long_kernel<T, V>
          <<<static_cast<unsigned>(std::min<int64_t>(a.rows, 2 * kNormBlocks)), kNormThreads, 0, s>>>(a);
    if (a.partial)
      layernorm_columns_kernel<T>
          <<<dim3((a.c + kNormThreads - 1) / kNormThreads, a.blocks), kNormThreads, 0, s>>>(a);
  }
}

template <typename T, int P, bool HALVES>
void rope(const RopeArgs &a, hipStream_t s) {
  rope_kernel<T, P, HALVES><<<static_cast<unsigned>((a.threads + 255) / 256), 256, 0, s>>>(a);
}

template <typename T>
void rope_any(const RopeArgs &a, int halves, int pairs, hipStream_t s) {
  if (halves) {
    if constexpr (sizeof(T) == 2)
      if (pairs == 8) return rope<T, 8, true>(a, s);
    if (pairs == 4) return rope<T, 4, true>(a, s);
    if (pairs == 2) return rope<T, 2, true>(a, s);
    return rope<T, 1, true>(a, s);
  }
  if constexpr (sizeof(T) == 2)
    if (pairs == 4) return rope<T, 4, false>(a, s);
  if (pairs == 2) return rope<T, 2, false>(a, s);
  return rope<T, 1, false>(a, s);
}

}  // namespace

int layernorm_bwd_blocks(int64_t rows) {
  // A workgroup's partial sums (2 c floats, written and read) against its rows
  // (3 c elements): at least 16 rows each, and no more than fill the chip.
  const int64_t want = (rows + 15) / 16;
  return static_cast<int>(std::min<int64_t>(std::max<int64_t>(want, 1), kNormBlocks));
}

int launch_layernorm_fwd(const NormArgs &a, int dtype, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == RT3D_F32) norm_fwd<float, 4>(a, s);
  else if (dtype == RT3D_BF16) norm_fwd<__bf16, 8>(a, s);
  else norm_fwd<_Float16, 8>(a, s);
  return hipGetLastError();
}

int launch_layernorm_bwd(const NormArgs &a, int dtype, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == RT3D_F32) norm_bwd<float, 4>(a, s);
  else if (dtype == RT3D_BF16) norm_bwd<__bf16, 8>(a, s);
  else norm_bwd<_Float16, 8>(a, s);
  if (a.partial)
    layernorm_finalize_kernel<<<(2 * a.c + kFinalCols - 1) / kFinalCols, kFinalCols * kFinalRuns, 0, s>>>(a);
  return hipGetLastError();
}

int launch_rope(const RopeArgs &a, int dtype, int halves, int pairs, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == RT3D_F32) rope_any<float>(a, halves, pairs, s);
  else if (dtype == RT3D_BF16) rope_any<__bf16>(a, halves, pairs, s);
  else rope_any<_Float16>(a, halves, pairs, s);
  return hipGetLastError();
}

}  // namespace rt3d
