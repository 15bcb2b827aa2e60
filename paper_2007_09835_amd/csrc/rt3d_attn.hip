// Differential attention on gfx950 (MI355X), forward.  Two softmax maps share
// the values: with S_m = scale q_m k_m^T over the visible keys and P_m its softmax,
//   o = P_1 v - lambda P_2 v,
// v twice as wide as a query vector.  Queries of the heads that share a key head
// are rows of one matrix, row r = query r / group of head r % group.

#include "rt3d_attn.h"

namespace rt3d {
namespace {

using namespace attn;

// One wave holds 32 rows and walks the keys once with the running maximum and
// sum of both maps.  S^T = K Q^T puts a row into a lane (and its other half), so
// the softmax needs one exchange between halves, and the probabilities are the
// second operand of O^T += V^T P^T where they stand: no trip through LDS.  Keys
// and values are staged by direct loads, two tiles deep.  Up to d = 64 a wave
// holds both maps, whose products share the value operands; beyond that their
// 2 x 32 x 256 results would take every accumulator, so two waves hold one map
// each of the same rows and meet at the end.
// ROWS: groups of 32 rows of a workgroup.
template <typename T, int D, int ROWS>
struct Fwd {
  static constexpr int kMaps = D > 64 ? 1 : 2;
  static constexpr int kWaves = ROWS * 2 / kMaps;
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kKeys = ROWS == 1 || D > 64 ? 32 : 64;
  static constexpr int kWidth = 2 * D;
  using KV = Tile<T, D, kKeys, kThreads>;
  static constexpr int kLds = 4 * KV::kBytes;
  static constexpr int kMinWaves = sizeof(T) == 2 || D <= 32 ? 2 : 1;
  // operands read ahead of their products: registers for them are left in 16 bits
  static constexpr bool kAhead = sizeof(T) == 2;
  // The transposing reads wait for every load under way: the next tile's loads
  // start behind the first ones of a tile that has more, else at once.
  static constexpr bool kLate = kKeys == 64;
  // Of the two waves of a SIMD one should multiply while the other is in its
  // softmax: the softmax goes first, then scores, then the products with v.  (8
  // clips of 4096 tokens, d 64: 772 us without, 740 with; d 128 838 and 831.  At d 32,
  // with three waves, 104 and 106: left alone there.)
  static constexpr bool kTurns = sizeof(T) == 2 && D > 32;
  static_assert(kMaps == 2 || ROWS * 32 * kWidth * 4 <= kLds, "the second maps' results fit");
};

// A row's reference is the maximum of its first 32 keys (or of the first 32 that hold
// a score above -inf), and no maximum is formed after that: a step whose probabilities
// against the reference add up to more than this (in a lane, 16 keys) is done again
// with a new one, everything before it scaled down.  P up to 2^8 fits every type, and
// steps after the first hardly ever get there where scores are alike along the keys.
// (8 clips of 4096 tokens, 8 heads, d 64: 705 us; scores that rise by 10 along the
// clip 746, by 160 932; a rise that repeats every step 1254.  8 clips of 1568, d 32: 95,
// 112, 163, 166.)
constexpr float kMost = 256.f;

template <typename T, int D, int ROWS, bool SPLIT>
__global__ __launch_bounds__((Fwd<T, D, ROWS>::kThreads), (Fwd<T, D, ROWS>::kMinWaves)) void attn_fwd_kernel(
    AttnArgs a) {
  using F = Fwd<T, D, ROWS>;
  using KV = typename F::KV;
  constexpr int kKeys = F::kKeys, kTiles = F::kWidth / 32, kMaps = F::kMaps;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lds_char *lds = (lds_char *)smem;

  Place here;
  if (!place(a, a.k_len, a.lk, here)) return;
  const int split = SPLIT ? here.split : 0, kvh = here.kvh, clip = here.clip;
  const int tile = a.tiles - 1 - here.rank;  // rows with most keys first

  const int q_len = clip_length(a.q_len, clip, a.lq), k_len = clip_length(a.k_len, clip, a.lk);
  const int rows = a.lq * a.group, used = q_len * a.group;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = uniform(static_cast<int>(threadIdx.x) >> 6);
  const int map0 = kMaps == 1 ? wave & 1 : 0;  // first map of this wave
  const int first = (tile * ROWS + wave * kMaps / 2) * 32, row = first + (lane & 31);
  const int query = row / a.group, head = kvh * a.group + (row - query * a.group);
  const bool in = row < used;
  const int limit = in ? visible(query, q_len, k_len, a.frame) : 0x7fffffff;

  // keys of the workgroup and of this wave (rows see at least as many as those before)
  const int last_block = min(used, (tile + 1) * ROWS * 32) - 1, last_wave = min(used, first + 32) - 1;
  int begin = 0, end = last_block < tile * ROWS * 32 ? 0 : visible(last_block / a.group, q_len, k_len, a.frame);
  const int wave_end = last_wave < first ? 0 : visible(last_wave / a.group, q_len, k_len, a.frame);
  const int whole = last_wave < first ? 0 : visible(first / a.group, q_len, k_len, a.frame);
  if (SPLIT) {
    begin = split * a.span;
    end = min(end, begin + a.span);
  }

  f32x16 acc[kMaps][kTiles] = {};
  float top[kMaps], sum[kMaps];
#pragma unroll
  for (int m = 0; m < kMaps; ++m) top[m] = -INFINITY, sum[m] = 0.f;

  if (begin < end) {
    Frag<T> q[kMaps][D / 16];
    {
      const T *p = static_cast<const T *>(a.q) + clip * a.q_batch + query * a.q_pitch +
                   (static_cast<int64_t>(head) * 2 + map0) * a.d;
#pragma unroll
      for (int m = 0; m < kMaps; ++m)
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          const int col = s * 16 + 8 * half;
          q[m][s] = in && col < a.d ? load_frag(p + m * a.d + col) : Frag<T>{};
        }
    }
    typename KV::Offsets k_off, v_off;
    KV::template offsets<true>(a.d, a.k_pitch, k_off);
    KV::template offsets<false>(a.d, a.v_pitch, v_off);
    const T *k = static_cast<const T *>(a.k) + clip * a.k_batch + static_cast<int64_t>(kvh) * 2 * a.d;
    const T *v = static_cast<const T *>(a.v) + clip * a.v_batch + static_cast<int64_t>(kvh) * 2 * a.d;
    auto stage = [&](int key, int buf) {
      const int n = min(kKeys, k_len - key);
      KV::stage(k + key * a.k_pitch, n, a.d, a.k_pitch, k_off, lds + buf * 2 * KV::kBytes);
      KV::stage(v + key * a.v_pitch, n, a.d, a.v_pitch, v_off, lds + (buf * 2 + 1) * KV::kBytes);
    };
    // (a second map's vectors begin a whole number of 16 blocks on: beyond d = 64)
    const unsigned k_lane = KV::lane_along() + map0 * D * KV::kEs, v_lane = KV::lane_across();
    using Scores = f32x16[kMaps];
    auto scores = [&](Scores &s, unsigned kt, int j) {
#pragma unroll
      for (int m = 0; m < kMaps; ++m)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) s[m] = Mma<T>::run(KV::along(kt, j, m * D + i * 16), q[m][i], s[m]);
    };
    auto hide = [&](Scores &s, int key) {
#pragma unroll
      for (int m = 0; m < kMaps; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key + result_row(i, half) >= limit) s[m][i] = -INFINITY;
    };
    // the reference, to the maximum so far (found: of rows that have one already, too)
    auto raise = [&](const Scores &s, bool found) {
#pragma unroll
      for (int m = 0; m < kMaps; ++m) {
        float most = s[m][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, s[m][i]);
        const float seen = half_max(most) * a.scale2;
        const float now = found || top[m] == -INFINITY ? fmaxf(top[m], seen) : top[m];
        const float by = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[m] - now);
        top[m] = now;
        sum[m] *= by;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[m][t][i] *= by;
      }
    };
    auto probabilities = [&](Scores &s, float (&part)[kMaps]) {
      bool over = false;
#pragma unroll
      for (int m = 0; m < kMaps; ++m) {
        const float ref = top[m] == -INFINITY ? 0.f : -top[m];
        part[m] = 0.f;  // short chains: the sum of a long row keeps its digits
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[m][i] = __builtin_amdgcn_exp2f(fmaf(s[m][i], a.scale2, ref));
          part[m] += s[m][i];
        }
        over |= part[m] > kMost;
      }
      return over;
    };
    stage(begin, 0);
    int buf = 0;
    bool start = true;  // some row of this wave has no reference yet
    for (int tile_key = begin; tile_key < end; tile_key += kKeys, buf ^= 1) {
      tile_barrier();  // this tile has landed, and the other buffer is read
      const unsigned kt = KV::at(k_lane, lds + buf * 2 * KV::kBytes), vt = KV::at(v_lane, lds + (buf * 2 + 1) * KV::kBytes);
      const bool more = tile_key + kKeys < end;
      if (!F::kLate && more) stage(tile_key + kKeys, buf ^ 1);
#pragma unroll
      for (int j = 0; j < kKeys; j += 32) {
        const int key = tile_key + j;
        if (key >= wave_end) {
          if (F::kLate && j == 0 && more) stage(tile_key + kKeys, buf ^ 1);
          break;
        }
        if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(1);
        f32x16 s[kMaps] = {};
        if constexpr (F::kAhead) {
          // keys' operands, D / 16 products ahead of their use
          constexpr int kN = kMaps * D / 16, kRing = D / 16 < 4 ? D / 16 : 4;
          Frag<T> f[kRing];
#pragma unroll
          for (int i = 0; i < kRing; ++i) f[i] = KV::along(kt, j, i * 16);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const int m = i / (D / 16);
            s[m] = Mma<T>::run(f[i % kRing], q[m][i % (D / 16)], s[m]);
            if (i + kRing < kN) f[i % kRing] = KV::along(kt, j, (i + kRing) * 16);
            __builtin_amdgcn_sched_barrier(0);
          }
        } else {
          scores(s, kt, j);
        }
        Frag<T> v0[kTiles];  // values of the first 16 keys, on their way during the softmax
        if constexpr (F::kAhead) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t) v0[t] = KV::across(vt, j, t * 32);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (F::kLate && j == 0 && more) stage(tile_key + kKeys, buf ^ 1);
        if (key + 32 > whole) hide(s, key);
        if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(2);
        const bool raised = start;
        if (raised) {
          raise(s, false);
          bool open = false;
#pragma unroll
          for (int m = 0; m < kMaps; ++m) {
            float all = s[m][0];  // -inf, or NaN: a row of NaN finds none and needs none
#pragma unroll
            for (int i = 1; i < 16; ++i) all += s[m][i];
            open |= top[m] == -INFINITY && all == -INFINITY;
          }
          start = __any(open && in && limit > begin);
        }
        float part[kMaps];
        bool over = probabilities(s, part);
        if (__builtin_expect(__any(over), 0)) {
#pragma unroll
          for (int m = 0; m < kMaps; ++m) s[m] = f32x16{};
          scores(s, kt, j);
          if (key + 32 > whole) hide(s, key);
          raise(s, true);
          probabilities(s, part);
        }
#pragma unroll
        for (int m = 0; m < kMaps; ++m) sum[m] += part[m];
        // Rounded to the layer's type for the product with v (half a step of
        // each probability); their sums keep 32 bits.
        Frag<T> p[kMaps][2];
#pragma unroll
        for (int m = 0; m < kMaps; ++m) p[m][0] = pack<T>(s[m], 0), p[m][1] = pack<T>(s[m], 8);
        Frag<T> v1[kTiles];
        if constexpr (F::kAhead) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int t = 0; t < kTiles; ++t) v1[t] = KV::across(vt, j + 16, t * 32);
        }
        if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            Frag<T> f;
            if constexpr (F::kAhead) f = h ? v1[t] : v0[t];
            else f = KV::across(vt, j + 16 * h, t * 32);
#pragma unroll
            for (int m = 0; m < kMaps; ++m) acc[m][t] = Mma<T>::run(f, p[m][h], acc[m][t]);
          }
      }
    }
  }

#pragma unroll
  for (int m = 0; m < kMaps; ++m) sum[m] = half_sum(sum[m]);
  if (SPLIT) {
    if (!in) return;
    const int64_t r = (static_cast<int64_t>(clip) * a.hk + kvh) * rows + row;
    const int64_t total = static_cast<int64_t>(a.n) * a.hk * rows;
    float *st = a.part + (split * total + r) * 4 + 2 * map0;
    float *out = a.part + a.splits * total * 4 + (split * total + r) * 4 * a.d + 2 * map0 * a.d;
#pragma unroll
    for (int m = 0; m < kMaps; ++m) {
      if (half == 0) {
        st[2 * m] = top[m];
        st[2 * m + 1] = sum[m];
      }
      if (sum[m] == 0.f) continue;  // no key here: nothing is read back
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = t * 32 + 8 * g + 4 * half;
          if (col < 2 * a.d)
            *reinterpret_cast<f32x4 *>(out + m * 2 * a.d + col) =
                f32x4{acc[m][t][4 * g], acc[m][t][4 * g + 1], acc[m][t][4 * g + 2], acc[m][t][4 * g + 3]};
        }
    }
    return;
  }

  // A map of a row that sees no key (or none with a score above -inf), and rows behind
  // the clip's end: zeros, and a logarithm of +inf, which makes every probability of
  // the backward pass zero.  (A sum of NaN is not zero: it goes into the row's results.)
  bool any[kMaps];
#pragma unroll
  for (int m = 0; m < kMaps; ++m) {
    any[m] = in && sum[m] != 0.f;
    const float inv = any[m] ? 1.f / sum[m] : 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][t][i] = any[m] ? acc[m][t][i] * inv : 0.f;
  }
  const float *handed = reinterpret_cast<const float *>(smem) + (wave >> 1) * 32 * F::kWidth + lane;
  if constexpr (kMaps == 1) {
    // the second map's wave hands its results to the first one's
    float *x = reinterpret_cast<float *>(smem) + (wave >> 1) * 32 * F::kWidth + lane;
    tile_barrier();
    if (map0) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(t * 16 + i) * 64] = acc[0][t][i];
    }
    tile_barrier();
  }
  if (row >= rows) return;
  const float lam = a.lam[head];
  T *o = static_cast<T *>(a.out) + clip * a.o_batch + query * a.o_pitch + static_cast<int64_t>(head) * 2 * a.d;
  T *o2 = static_cast<T *>(a.out2) + ((static_cast<int64_t>(clip) * a.lq + query) * a.hq + head) * 2 * a.d;
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  };
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = t * 32 + 8 * g + 4 * half;
      if (col >= 2 * a.d) continue;
      Four x, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * g + e;
        const float second = kMaps == 2 ? acc[kMaps - 1][t][i] : map0 ? acc[0][t][i] : handed[(t * 16 + i) * 64];
        x.v[e] = static_cast<T>(acc[0][t][i] - lam * second);
        y.v[e] = static_cast<T>(second);
      }
      if (!map0) *reinterpret_cast<Four *>(o + col) = x;
      if (a.out2 && map0 == kMaps % 2) *reinterpret_cast<Four *>(o2 + col) = y;
    }
  if (a.lse && half == 0) {
    const int64_t stat = (static_cast<int64_t>(clip) * a.hq + head) * a.lq + query;
#pragma unroll
    for (int m = 0; m < kMaps; ++m)
      a.lse[(map0 + m) * static_cast<int64_t>(a.n) * a.hq * a.lq + stat] = any[m] ? top[m] + log2f(sum[m]) : INFINITY;
  }
}

// Joins the splits of a row in their order.  SHARE waves per row: each finds the
// splits' weights (a lane per split), sums its share of them with half of its
// lanes per map and four columns per lane, and the shares meet in LDS.
constexpr int kMaxSplits = 256;
template <typename T, int SHARE>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  constexpr int kPer = kMaxSplits / 64;
  __shared__ f32x4 shared[SHARE > 1 ? SHARE - 1 : 1][64];
  const int rows = a.lq * a.group, lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x) >> 6);
  const int64_t total = static_cast<int64_t>(a.n) * a.hk * rows;
  const int64_t r = SHARE > 1 ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * 4 + wave;
  const int share = SHARE > 1 ? wave : 0;
  if (r >= total) return;
  const int row = static_cast<int>(r % rows);
  const int64_t pair = r / rows;
  const int kvh = static_cast<int>(pair % a.hk), clip = static_cast<int>(pair / a.hk);
  const int query = row / a.group, head = kvh * a.group + (row - query * a.group);
  const bool in = query < clip_length(a.q_len, clip, a.lq);
  float weight[2][kPer], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
  f32x4 st[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int s = i * 64 + lane;
    st[i] = f32x4{-INFINITY, 0.f, -INFINITY, 0.f};
    if (in && s < a.splits) st[i] = *reinterpret_cast<const f32x4 *>(a.part + (s * total + r) * 4);
#pragma unroll
    for (int m = 0; m < 2; ++m) top[m] = fmaxf(top[m], st[i][2 * m]);
  }
#pragma unroll
  for (int w = 32; w > 0; w >>= 1)
#pragma unroll
    for (int m = 0; m < 2; ++m) top[m] = fmaxf(top[m], __shfl_xor(top[m], w, 64));
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      // a split without keys has weight zero: its results were not written and are not used
      weight[m][i] = st[i][2 * m + 1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[i][2 * m] - top[m]);
      sum[m] += weight[m][i] * st[i][2 * m + 1];
    }
#pragma unroll
  for (int w = 32; w > 0; w >>= 1)
#pragma unroll
    for (int m = 0; m < 2; ++m) sum[m] += __shfl_xor(sum[m], w, 64);
  const float lam = a.lam[head];
  T *o = static_cast<T *>(a.out) + clip * a.o_batch + query * a.o_pitch + static_cast<int64_t>(head) * 2 * a.d;
  T *o2 = static_cast<T *>(a.out2) + ((static_cast<int64_t>(clip) * a.lq + query) * a.hq + head) * 2 * a.d;
  const int m = lane >> 5;
  const float total_sum = m ? sum[1] : sum[0], total_top = m ? top[1] : top[0];
  const bool any = in && total_sum != 0.f;
  const float *part = a.part + a.splits * total * 4 + r * 4 * a.d + m * 2 * a.d;
  const int64_t step = total * 4 * a.d;
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  };
  for (int c0 = 0; c0 < 2 * a.d; c0 += 128) {
    const int col = c0 + (lane & 31) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (in) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int n = min(64, a.splits - i * 64);
        for (int s0 = share; s0 < n; s0 += 8 * SHARE) {
          f32x4 x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {  // eight loads in flight
            const int s = min(s0 + j * SHARE, n - 1);
            x[j] = *reinterpret_cast<const f32x4 *>(part + (i * 64 + s) * step + (col < 2 * a.d ? col : 0));
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int s = s0 + j * SHARE;
            const float w0 = __shfl(weight[0][i], s, 64), w1 = __shfl(weight[1][i], s, 64), by = m ? w1 : w0;
            if (s < n && by != 0.f) {  // (one map's weight may vanish alone)
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] += by * x[j][e];
            }
          }
        }
      }
    }
    if constexpr (SHARE > 1) {
      __syncthreads();
      if (share) shared[share - 1][lane] = v;
      __syncthreads();
      if (share) continue;
#pragma unroll
      for (int s = 0; s < SHARE - 1; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += shared[s][lane][e];
    }
    Four x, y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float mine = any ? v[e] / total_sum : 0.f, other = __shfl_xor(mine, 32, 64);
      x.v[e] = static_cast<T>(mine - lam * other);
      y.v[e] = static_cast<T>(mine);
    }
    if (col >= 2 * a.d) continue;
    if (m == 0) *reinterpret_cast<Four *>(o + col) = x;
    if (m == 1 && a.out2) *reinterpret_cast<Four *>(o2 + col) = y;
  }
  if (a.lse && share == 0 && (lane & 31) == 0) {
    const int64_t at = (static_cast<int64_t>(clip) * a.hq + head) * a.lq + query;
    a.lse[m * static_cast<int64_t>(a.n) * a.hq * a.lq + at] = any ? total_top + log2f(total_sum) : INFINITY;
  }
}

template <typename T, int D, int ROWS, bool SPLIT>
int fwd(const AttnArgs &a, hipStream_t s) {
  using F = Fwd<T, D, ROWS>;
  static_assert(F::kThreads == attn_fwd_threads(D, ROWS), "what the host checks the launch for");
  const int e = allow_lds<attn_fwd_kernel<T, D, ROWS, SPLIT>>(F::kLds);
  if (e != hipSuccess) return e;
  attn_fwd_kernel<T, D, ROWS, SPLIT><<<grid_of(a.blocks), F::kThreads, F::kLds, s>>>(a);
  if (SPLIT) {
    const int64_t rows = static_cast<int64_t>(a.n) * a.hk * a.lq * a.group;
    // four waves share a row's splits where there are more than a few
    if (a.splits > 16) attn_join_kernel<T, 4><<<static_cast<unsigned>(rows), 256, 0, s>>>(a);
    else attn_join_kernel<T, 1><<<static_cast<unsigned>((rows + 3) / 4), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, int D>
int fwd_shape(const AttnArgs &a, int rows, hipStream_t s) {
  constexpr int kMost = attn_row_groups(D);
  if (rows == 1) return a.splits > 1 ? fwd<T, D, 1, true>(a, s) : fwd<T, D, 1, false>(a, s);
  return a.splits > 1 ? fwd<T, D, kMost, true>(a, s) : fwd<T, D, kMost, false>(a, s);
}

template <typename T>
int fwd_type(const AttnArgs &a, int rows, hipStream_t s) {
  if (a.d <= 32) return fwd_shape<T, 32>(a, rows, s);
  if (a.d <= 64) return fwd_shape<T, 64>(a, rows, s);
  return fwd_shape<T, 128>(a, rows, s);
}

}  // namespace

int launch_attn_fwd(const AttnArgs &a, int dtype, int rows, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == RT3D_F32) return fwd_type<float>(a, rows, s);
  if (dtype == RT3D_BF16) return fwd_type<__bf16>(a, rows, s);
  return fwd_type<_Float16>(a, rows, s);
}

}  // namespace rt3d
