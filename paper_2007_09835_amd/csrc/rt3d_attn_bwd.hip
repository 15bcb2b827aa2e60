// Differential attention on gfx950 (MI355X), backward.  With P_m the softmax maps,
// A_m the row sums of P_m dP and dP = do v^T:
//   dS_1 = P_1 (dP - A_1),  dS_2 = -lambda P_2 (dP - A_2),
//   dq_m = scale dS_m k_m,  dk_m = scale dS_m^T q_m,  dv = (P_1 - lambda P_2)^T do,
//   dlambda = -sum of P_2 dP.
// The probabilities come back from the scores and the logarithms that the
// forward pass left.  A_m = do . o_m is formed from o and the second map's output.
// Two kernels, each owning what it sums, so no result depends on an order of
// arrival: one walks the keys for its query rows, one the queries for its keys.

#include "rt3d_attn.h"

namespace rt3d {
namespace {

using namespace attn;

template <typename T, int D, int WAVES>
struct Dq {
  static constexpr int kKeys = WAVES == 1 || D > 64 || sizeof(T) == 4 ? 32 : 64;
  static constexpr int kThreads = 64 * WAVES;
  using KV = Tile<T, D, kKeys, kThreads>;
  static constexpr int kLds = 4 * KV::kBytes;
  static constexpr int kMinWaves = sizeof(T) == 2 && D <= 64 ? 2 : 1;
  // 32-bit output gradients of 256 columns beside the queries pass the register
  // file: they are read again for every step, from L1.
  static constexpr bool kHoldG = sizeof(T) == 2 || D <= 64;
  // As in the forward pass, one of a SIMD's two waves should multiply while the
  // other forms probabilities, which go first, then scores, then the products of
  // the gradient.  (2 clips of 6272 tokens, 8 heads, d 64, causal: 369 us without, 340.)
  static constexpr bool kTurns = sizeof(T) == 2;
};

// Rows of queries as in the forward pass (a lane holds a row): S^T = K Q^T and
// dP^T = V dO^T leave dS^T where the product dQ^T += K^T dS^T takes it.
// SPLIT: the keys are split over workgroups, which leave 32-bit partial gradients.
template <typename T, int D, int WAVES, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, (Dq<T, D, WAVES>::kMinWaves)) void attn_dq_kernel(AttnArgs a) {
  using F = Dq<T, D, WAVES>;
  using KV = typename F::KV;
  constexpr int kKeys = F::kKeys;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lds_char *lds = (lds_char *)smem;

  Place here;
  if (!place(a, a.k_len, a.lk, here)) return;
  const int split = SPLIT ? here.split : 0, kvh = here.kvh, clip = here.clip;
  const int tile = a.tiles - 1 - here.rank;  // rows with most keys first
  const int q_len = clip_length(a.q_len, clip, a.lq), k_len = clip_length(a.k_len, clip, a.lk);
  const int rows = a.lq * a.group, used = q_len * a.group;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = uniform(static_cast<int>(threadIdx.x) >> 6);
  const int first = (tile * WAVES + wave) * 32, row = first + (lane & 31);
  const int query = row / a.group, head = kvh * a.group + (row - query * a.group);
  const bool in = row < used;
  const int limit = in ? visible(query, q_len, k_len, a.frame) : 0x7fffffff;
  const int last_block = min(used, (tile + 1) * WAVES * 32) - 1, last_wave = min(used, first + 32) - 1;
  const int all = last_block < tile * WAVES * 32 ? 0 : visible(last_block / a.group, q_len, k_len, a.frame);
  const int begin = SPLIT ? split * a.span : 0, end = SPLIT ? min(all, begin + a.span) : all;
  const int wave_end = last_wave < first ? 0 : visible(last_wave / a.group, q_len, k_len, a.frame);
  const int whole = last_wave < first ? 0 : visible(first / a.group, q_len, k_len, a.frame);

  const int64_t map = static_cast<int64_t>(a.n) * a.hq * a.lq;
  const int64_t stat = (static_cast<int64_t>(clip) * a.hq + head) * a.lq + query;
  const float lam = in ? a.lam[head] : 0.f;
  f32x16 acc[2][D / 32] = {};
  float dl = 0.f;

  if (begin < end) {
    Frag<T> q[2][D / 16], g[F::kHoldG ? 2 * D / 16 : 1];
    float lse[2] = {INFINITY, INFINITY}, mean[2] = {0.f, 0.f};
    const T *go = static_cast<const T *>(a.d_o) + clip * a.do_batch + query * a.do_pitch +
                  static_cast<int64_t>(head) * 2 * a.d;
    auto grad_frag = [&](int s) {
      const int col = s * 16 + 8 * half;
      return in && col < 2 * a.d ? load_frag(go + col) : Frag<T>{};
    };
    {
      const T *p = static_cast<const T *>(a.q) + clip * a.q_batch + query * a.q_pitch +
                   static_cast<int64_t>(head) * 2 * a.d;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          const int col = s * 16 + 8 * half;
          q[m][s] = in && col < a.d ? load_frag(p + m * a.d + col) : Frag<T>{};
        }
      const T *o = static_cast<const T *>(a.o) + clip * a.o_batch + query * a.o_pitch +
                   static_cast<int64_t>(head) * 2 * a.d;
      const T *o2 = static_cast<const T *>(a.o2) +
                    ((static_cast<int64_t>(clip) * a.lq + query) * a.hq + head) * 2 * a.d;
#pragma unroll
      for (int s = 0; s < 2 * D / 16; ++s) {
        const int col = s * 16 + 8 * half;
        const bool get = in && col < 2 * a.d;
        const Frag<T> grad = grad_frag(s);
        if constexpr (F::kHoldG) g[s] = grad;
        const Frag<T> x = get ? load_frag(o + col) : Frag<T>{}, y = get ? load_frag(o2 + col) : Frag<T>{};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          mean[0] += static_cast<float>(grad[e]) * static_cast<float>(x[e]);
          mean[1] += static_cast<float>(grad[e]) * static_cast<float>(y[e]);
        }
      }
      mean[1] = half_sum(mean[1]);
      mean[0] = half_sum(mean[0]) + lam * mean[1];
      if (in) {
        lse[0] = a.lse[stat];
        lse[1] = a.lse[map + stat];
        if (half == 0 && begin == 0) {
          a.rowstat[stat] = mean[0];
          a.rowstat[map + stat] = mean[1];
        }
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
    const unsigned along = KV::lane_along(), across = KV::lane_across();
    auto gradients = [&](unsigned vt, int j) {  // dP of 32 keys
      f32x16 dp = {};
      if constexpr (sizeof(T) == 2) {
        dp = chain<T, 2 * D / 16>([&](int i) { return KV::along(vt, j, i * 16); }, [&](int i) { return g[i]; }, dp);
      } else {
#pragma unroll
        for (int i = 0; i < 2 * D / 16; ++i) {
          Frag<T> b;
          if constexpr (F::kHoldG) b = g[i];
          else b = grad_frag(i);
          dp = Mma<T>::run(KV::along(vt, j, i * 16), b, dp);
        }
      }
      return dp;
    };
    auto scores = [&](unsigned kt, int key, int j, int m, bool masked) {
      f32x16 s = {};
      if constexpr (sizeof(T) == 2) {
        s = chain<T, D / 16>([&](int i) { return KV::along(kt, j, m * D + i * 16); }, [&](int i) { return q[m][i]; },
                             s);
      } else {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) s = Mma<T>::run(KV::along(kt, j, m * D + i * 16), q[m][i], s);
      }
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key + j + result_row(i, half) >= limit) s[i] = -INFINITY;
      }
      return s;
    };
    stage(begin, 0);
    // Rows of few keys, all of them in the first tile: the roundings of o and of the
    // probabilities in it do not average out, and a row sum formed from o is as far off
    // as the differences dP - A are small (bf16, d 64, two keys, normal inputs: dq is
    // 0.45% off in the median and 6% in one row of twenty, with values around 3 1.3% and
    // 21%; with exact sums 0.2% and 0.35%). One tile more of work sums P dP itself,
    // whatever the workgroup's other rows see.
    const int first_block = visible(tile * WAVES * 32 / a.group, q_len, k_len, a.frame);
    if (begin == 0 && first_block <= kKeys) {
      tile_barrier();
      const unsigned kt = KV::at(along, lds), vt = KV::at(along, lds + KV::kBytes);
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kKeys; j += 32) {
        if (j >= wave_end || whole > kKeys) break;
        const f32x16 dp = gradients(vt, j);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const f32x16 s = scores(kt, 0, j, m, true);
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[m] += __builtin_amdgcn_exp2f(fmaf(s[i], a.scale2, -lse[m])) * dp[i];
        }
      }
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        sum[m] = half_sum(sum[m]);
        if (limit <= kKeys) {
          mean[m] = sum[m];
          if (half == 0) a.rowstat[m * map + stat] = mean[m];
        }
      }
    }
    int buf = 0;
    for (int key = begin; key < end; key += kKeys, buf ^= 1) {
      tile_barrier();
      if (key + kKeys < end) stage(key + kKeys, buf ^ 1);
      if (key >= wave_end) continue;
      const lds_char *tile_k = lds + buf * 2 * KV::kBytes;
      const unsigned kt = KV::at(along, tile_k), vt = KV::at(along, tile_k + KV::kBytes), kc = KV::at(across, tile_k);
      const bool masked = key + kKeys > whole;
#pragma unroll
      for (int j = 0; j < kKeys; j += 32) {
        if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(1);
        const f32x16 dp = gradients(vt, j);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(1);
          f32x16 s = scores(kt, key, j, m, masked);
          if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(2);
          float part = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale2, -lse[m]));
            if (m) part += p * dp[i];  // short chains: the sum over a long row keeps its digits
            s[i] = p * (dp[i] - mean[m]);
          }
          if (m) dl += part;
          const Frag<T> lo = pack<T>(s, 0), hi = pack<T>(s, 8);
          if constexpr (F::kTurns) __builtin_amdgcn_s_setprio(0);
#pragma unroll
          for (int t = 0; t < D / 32; ++t) {
            acc[m][t] = Mma<T>::run(KV::across(kc, j, m * D + t * 32), lo, acc[m][t]);
            acc[m][t] = Mma<T>::run(KV::across(kc, j + 16, m * D + t * 32), hi, acc[m][t]);
          }
        }
      }
    }
  }
  if (row >= rows) return;
  dl = half_sum(in ? dl : 0.f);  // (rows behind the clip's end meet keys, which may be infinite)
  if (half == 0) {
    a.rowstat[(2 + split) * map + stat] = dl;
    if (begin == 0 && end <= 0) a.rowstat[stat] = a.rowstat[map + stat] = 0.f;
  }
  if (!a.dq) return;
  // the softmax of a single key does not move, and rows behind the clip's end have none
  if (!in || limit <= 1) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < D / 32; ++t) acc[m][t] = f32x16{};
  }
  if constexpr (SPLIT) {
    float *p = a.part + (split * map + (static_cast<int64_t>(clip) * a.lq + query) * a.hq + head) * 2 * a.d;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float by = m ? -lam * a.scale : a.scale;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = t * 32 + 8 * r + 4 * half;
          if (col < a.d)
            *reinterpret_cast<f32x4 *>(p + m * a.d + col) =
                f32x4{acc[m][t][4 * r] * by, acc[m][t][4 * r + 1] * by, acc[m][t][4 * r + 2] * by,
                      acc[m][t][4 * r + 3] * by};
        }
    }
    return;
  }
  T *dq = static_cast<T *>(a.dq) + clip * a.dq_batch + query * a.dq_pitch + static_cast<int64_t>(head) * 2 * a.d;
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  };
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const float by = m ? -lam * a.scale : a.scale;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = t * 32 + 8 * r + 4 * half;
        if (col >= a.d) continue;
        Four x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] = static_cast<T>(acc[m][t][4 * r + e] * by);
        *reinterpret_cast<Four *>(dq + m * a.d + col) = x;
      }
  }
}

// dlambda of a head, by a workgroup of 256: its rows' sums over the clips and
// splits, in a fixed order.
__device__ __forceinline__ void sum_dlam(const AttnArgs &a, int head, float *lds) {
  const float *p = a.rowstat + 2 * static_cast<int64_t>(a.n) * a.hq * a.lq;
  const unsigned len = a.lq, total = static_cast<unsigned>(a.stat_splits) * a.n * len;  // below 2^31 rows
  float s = 0.f;
#pragma unroll 8
  for (unsigned i = threadIdx.x; i < total; i += 256) {
    const unsigned part = i / len;
    s += p[(static_cast<int64_t>(part) * a.hq + head) * len + (i - part * len)];
  }
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) s += __shfl_xor(s, w, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.dlam[head] = 0.f - ((lds[0] + lds[1]) + (lds[2] + lds[3]));
}

// A lane holds a key: S = Q K^T and dP = dO V^T with the keys and values in
// registers leave P and dS where dV^T += dO^T P and dK^T += Q^T dS take them.  The
// heads of a key head's group follow one another and add to the same results.
template <typename T, int D, int WAVES>
struct Dkv {
  static constexpr int kRows = 32;
  static constexpr int kThreads = 64 * WAVES;
  using Q = Tile<T, D, kRows, kThreads>;
  static constexpr int kStat = 4 * 64 * 4;  // logarithms and row sums of the tile's rows
  static constexpr int kMinWaves = sizeof(T) == 2 && D <= 64 ? 2 : 1;
  // Values stay in registers, and keys where both fit beside their gradients;
  // otherwise keys wait in LDS.  32-bit values of 256 columns (and their keys)
  // pass both: they are read again for every tile, from L1.
  static constexpr bool kHoldV = sizeof(T) == 2 || D <= 64, kHoldK = D <= 32, kLdsK = !kHoldK && kHoldV;
  // Operands read ahead of their products and waves that take turns, as in dq, where
  // registers are left for it: in 16 bits, but not with both gradients at d = 64.  (4
  // clips of 4096 tokens, 4 heads, d 32: 256 us without, 225; 2 clips, 8 heads, d 128: dk
  // 783 and 724, dv 574 and 541.  At d 64 it spilled and cost 3%.)
  static constexpr bool kAhead = sizeof(T) == 2 && (D <= 32 || D > 64);
  // Beyond d = 64 both gradients (2 x 32 x 256 results) would take every
  // accumulator and leave none for scores: the kernel runs once for each.
  static constexpr bool kApart = D > 64;
  using K = Tile<T, D, 32 * WAVES, kThreads>;
  static constexpr int kBuffer = 2 * Q::kBytes + kStat;
  static constexpr int kLds = 2 * kBuffer + (kLdsK ? K::kBytes : 0);
};

// SPLIT: the query tiles of a key head (its group's heads, one after another) are
// split over workgroups, which leave 32-bit partial gradients.  DK, DV: which
// gradients this launch makes.
template <typename T, int D, int WAVES, bool SPLIT, bool DK, bool DV>
__global__ __launch_bounds__(64 * WAVES, (Dkv<T, D, WAVES>::kMinWaves)) void attn_dkv_kernel(AttnArgs a) {
  using F = Dkv<T, D, WAVES>;
  using Q = typename F::Q;
  constexpr int kRows = F::kRows;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lds_char *lds = (lds_char *)smem;

  // the last workgroups add up dlambda, which needs no launch of its own then
  if (blockIdx.x >= gridDim.x - a.dlam_blocks) {
    sum_dlam(a, static_cast<int>(blockIdx.x - (gridDim.x - a.dlam_blocks)), reinterpret_cast<float *>(smem));
    return;
  }
  Place here;
  if (!place(a, a.q_len, a.lq, here)) return;
  const int split = SPLIT ? here.split : 0, kvh = here.kvh, clip = here.clip;
  const int tile = here.rank;  // keys that most queries see first
  const int q_len = clip_length(a.q_len, clip, a.lq), k_len = clip_length(a.k_len, clip, a.lk);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = uniform(static_cast<int>(threadIdx.x) >> 6);
  const int key_block = tile * WAVES * 32, key_wave = key_block + wave * 32, key = key_wave + (lane & 31);
  const bool in = key < k_len;
  // first query that sees a key: the one that stands where the key's frame begins
  auto first_query = [&](int k) { return a.frame ? k / a.frame * a.frame - (k_len - q_len) : 0; };
  const int from = first_query(key), from_wave = first_query(key_wave);
  // queries whose softmax has one key: all of a clip with one, or the one that
  // stands at the first key where every token is a frame (none if negative)
  const bool single_all = k_len == 1;
  const int single = a.frame == 1 ? q_len - k_len : -1;

  f32x16 dk[2][DK ? D / 32 : 1] = {}, dv[DV ? 2 * D / 32 : 1] = {};
  const int begin = max(0, first_query(key_block)) / kRows * kRows;

  // query tiles that see the workgroup's keys, a group's heads after one another,
  // and this split's share of them
  const int per_head = key_block < k_len && begin < q_len ? (q_len - begin + kRows - 1) / kRows : 0;
  const int total = per_head * a.group;
  const int from_tile = SPLIT ? static_cast<int>(static_cast<int64_t>(total) * split / a.splits) : 0;
  const int to_tile = SPLIT ? static_cast<int>(static_cast<int64_t>(total) * (split + 1) / a.splits) : total;

  if (from_tile < to_tile) {
    const T *k = static_cast<const T *>(a.k) + clip * a.k_batch + (in ? key : 0) * a.k_pitch +
                 static_cast<int64_t>(kvh) * 2 * a.d;
    const T *v = static_cast<const T *>(a.v) + clip * a.v_batch + (in ? key : 0) * a.v_pitch +
                 static_cast<int64_t>(kvh) * 2 * a.d;
    auto key_frag = [&](int m, int s) {
      const int col = s * 16 + 8 * half;
      return in && col < a.d ? load_frag(k + m * a.d + col) : Frag<T>{};
    };
    auto value_frag = [&](int s) {
      const int col = s * 16 + 8 * half;
      return in && col < 2 * a.d ? load_frag(v + col) : Frag<T>{};
    };
    Frag<T> kf[F::kHoldK ? 2 : 1][F::kHoldK ? D / 16 : 1], vf[F::kHoldV && DK ? 2 * D / 16 : 1];
    if constexpr (F::kHoldK) {
#pragma unroll
      for (int s = 0; s < D / 16; ++s) kf[0][s] = key_frag(0, s), kf[1][s] = key_frag(1, s);
    }
    if constexpr (F::kHoldV && DK) {
#pragma unroll
      for (int s = 0; s < 2 * D / 16; ++s) vf[s] = value_frag(s);
    }
    lds_char *keys = lds + 2 * F::kBuffer;
    if constexpr (F::kLdsK) {
      typename F::K::Offsets k_off;
      F::K::template offsets<true>(a.d, a.k_pitch, k_off);
      F::K::stage(static_cast<const T *>(a.k) + clip * a.k_batch + key_block * a.k_pitch +
                      static_cast<int64_t>(kvh) * 2 * a.d,
                  min(32 * WAVES, k_len - key_block), a.d, a.k_pitch, k_off, keys);
    }
    typename Q::Offsets q_off, g_off;
    Q::template offsets<true>(a.d, a.q_pitch, q_off);
    Q::template offsets<false>(a.d, a.do_pitch, g_off);
    const int64_t map = static_cast<int64_t>(a.n) * a.hq * a.lq;
    const T *q = static_cast<const T *>(a.q) + clip * a.q_batch;
    const T *go = static_cast<const T *>(a.d_o) + clip * a.do_batch;
    // tile t: rows of head t / per_head from begin + t % per_head * kRows on
    int head = from_tile / per_head, row0 = begin + (from_tile - head * per_head) * kRows;
    int st_head = head, st_row = row0;  // of the tile to be staged next
    auto stage = [&](int buf) {
      const int head = kvh * a.group + st_head, n = min(kRows, q_len - st_row);
      lds_char *to = lds + buf * F::kBuffer;
      Q::stage(q + st_row * a.q_pitch + static_cast<int64_t>(head) * 2 * a.d, n, a.d, a.q_pitch, q_off, to);
      Q::stage(go + st_row * a.do_pitch + static_cast<int64_t>(head) * 2 * a.d, n, a.d, a.do_pitch, g_off,
               to + Q::kBytes);
      // logarithms of both maps, then row sums: one row of 64 lanes each
#pragma unroll
      for (int i = 0; i < 4 / (WAVES < 4 ? WAVES : 4); ++i) {
        const int which = i * WAVES + wave;
        const int64_t at = (which & 1) * map + (static_cast<int64_t>(clip) * a.hq + head) * a.lq + st_row;
        const float *src = (which & 2 ? a.rowstat : a.lse) + at;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(src), 0, n * 4, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            r, (__attribute__((address_space(3))) void *)(to + 2 * Q::kBytes + which * 256), 4, lane * 4, 0, 0, 0);
      }
      if ((st_row += kRows) >= q_len) {
        st_row = begin;
        ++st_head;
      }
    };
    const unsigned along = Q::lane_along(), across = Q::lane_across();
    unsigned key_lane = 0;
    if constexpr (F::kLdsK) key_lane = F::K::lane_along() + wave * 32 * F::K::kRowBytes;
    stage(0);
    int buf = 0;
    for (int t = from_tile; t < to_tile; ++t, buf ^= 1) {
      tile_barrier();
      if (t + 1 < to_tile) stage(buf ^ 1);
      const float lam = a.lam[kvh * a.group + head];
      const int at = row0;
      if ((row0 += kRows) >= q_len) {
        row0 = begin;
        ++head;
      }
      // no row of the tile sees a key of this wave, or it has none
      if (at + kRows <= from_wave || key_wave >= k_len) continue;
      const lds_char *tile_q = lds + buf * F::kBuffer, *tile_g = tile_q + Q::kBytes, *st = tile_g + Q::kBytes;
      const unsigned qt = Q::at(along, tile_q), gt = Q::at(along, tile_g);
      const unsigned qc = Q::at(across, tile_q), gc = Q::at(across, tile_g);
      unsigned kt = 0;
      if constexpr (F::kLdsK) kt = F::K::at(key_lane, keys);
      // some pair of the tile is masked, or some row has a single key
      const bool masked = a.frame && at < first_query(min(key_wave + 31, k_len - 1));
      const bool lone = key_wave == 0 && (single_all || (single >= at && single < at + kRows));
      f32x16 dp = {}, pv;
      if constexpr (F::kAhead && DK) {
        __builtin_amdgcn_s_setprio(1);
        dp = chain<T, 2 * D / 16>([&](int i) { return Q::along(gt, 0, i * 16); }, [&](int i) { return vf[i]; }, dp);
      } else if constexpr (DK) {
#pragma unroll
        for (int i = 0; i < 2 * D / 16; ++i) {
          Frag<T> b;
          if constexpr (F::kHoldV) b = vf[i];
          else b = value_frag(i);
          dp = Mma<T>::run(Q::along(gt, 0, i * 16), b, dp);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        f32x16 s = {};
        Frag<T> qn[2][D / 32];  // queries of dk's products, on their way during the probabilities
        if constexpr (F::kAhead) {
          __builtin_amdgcn_s_setprio(1);
          auto queries = [&](int i) { return Q::along(qt, 0, m * D + i * 16); };
          if constexpr (F::kHoldK) s = chain<T, D / 16>(queries, [&](int i) { return kf[m][i]; }, s);
          else s = chain_both<T, D / 16>(queries, [&](int i) { return F::K::along(kt, 0, m * D + i * 16); }, s);
#pragma unroll
          for (int h = 0; DK && h < 2; ++h)
#pragma unroll
            for (int c = 0; c < D / 32; ++c) qn[h][c] = Q::across(qc, 16 * h, m * D + c * 32);
          __builtin_amdgcn_sched_barrier(0);
          __builtin_amdgcn_s_setprio(2);
        } else {
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            Frag<T> b;
            if constexpr (F::kHoldK) b = kf[m][i];
            else if constexpr (F::kLdsK) b = F::K::along(kt, 0, m * D + i * 16);
            else b = key_frag(m, i);
            s = Mma<T>::run(Q::along(qt, 0, m * D + i * 16), b, s);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (at + result_row(i, half) < from) s[i] = -INFINITY;
        }
        // rows behind the clip's end are zeros, which an infinite key would turn into NaN
        if (__builtin_expect(at + kRows > q_len, 0)) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (at + result_row(i, half) >= q_len) s[i] = -INFINITY;
        }
        const float by = m ? -lam : 1.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4 lse = *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(
              st + m * 256 + (8 * r + 4 * half) * 4);
          const f32x4 mean = *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(
              st + (2 + m) * 256 + (8 * r + 4 * half) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * r + e;
            const float p = by * __builtin_amdgcn_exp2f(fmaf(s[i], a.scale2, -lse[e]));
            if (DV) pv[i] = m ? pv[i] + p : p;
            s[i] = p * (dp[i] - mean[e]);
          }
        }
        if constexpr (!DK) continue;
        if (lone) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (single_all || at + result_row(i, half) == single) s[i] = 0.f;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Frag<T> ds = pack<T>(s, 8 * h);
          if constexpr (F::kAhead) __builtin_amdgcn_s_setprio(0);
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            if constexpr (!F::kAhead) qn[h][c] = Q::across(qc, 16 * h, m * D + c * 32);
            dk[m][c] = Mma<T>::run(qn[h][c], ds, dk[m][c]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int h = 0; DV && h < 2; ++h) {
        const Frag<T> p = pack<T>(pv, 8 * h);
#pragma unroll
        for (int c = 0; c < 2 * D / 32; ++c) dv[c] = Mma<T>::run(Q::across(gc, 16 * h, c * 32), p, dv[c]);
      }
    }
  }
  if (key >= a.lk) return;
  if constexpr (SPLIT) {
    float *p = a.part + ((split * static_cast<int64_t>(a.n) + clip) * a.lk + key) * a.hk * 4 * a.d +
               static_cast<int64_t>(kvh) * 4 * a.d;
#pragma unroll
    for (int m = 0; DK && m < 2; ++m)
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = t * 32 + 8 * r + 4 * half;
          if (col < a.d)
            *reinterpret_cast<f32x4 *>(p + m * a.d + col) =
                f32x4{dk[m][t][4 * r] * a.scale, dk[m][t][4 * r + 1] * a.scale, dk[m][t][4 * r + 2] * a.scale,
                      dk[m][t][4 * r + 3] * a.scale};
        }
#pragma unroll
    for (int t = 0; DV && t < 2 * D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = t * 32 + 8 * r + 4 * half;
        if (col < 2 * a.d)
          *reinterpret_cast<f32x4 *>(p + 2 * a.d + col) =
              f32x4{dv[t][4 * r], dv[t][4 * r + 1], dv[t][4 * r + 2], dv[t][4 * r + 3]};
      }
    return;
  }
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  };
  if (DK && a.dk) {
    T *p = static_cast<T *>(a.dk) + clip * a.dk_batch + key * a.dk_pitch + static_cast<int64_t>(kvh) * 2 * a.d;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = t * 32 + 8 * r + 4 * half;
          if (col >= a.d) continue;
          Four x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x.v[e] = static_cast<T>(in ? dk[m][t][4 * r + e] * a.scale : 0.f);
          *reinterpret_cast<Four *>(p + m * a.d + col) = x;
        }
  }
  if (DV && a.dv) {
    T *p = static_cast<T *>(a.dv) + clip * a.dv_batch + key * a.dv_pitch + static_cast<int64_t>(kvh) * 2 * a.d;
#pragma unroll
    for (int t = 0; t < 2 * D / 32; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int col = t * 32 + 8 * r + 4 * half;
        if (col >= 2 * a.d) continue;
        Four x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] = static_cast<T>(in ? dv[t][4 * r + e] : 0.f);
        *reinterpret_cast<Four *>(p + col) = x;
      }
  }
}

// Adds up the splits' partial gradients in their order: a thread per four columns.
// KEYS: dk and dv ([n][lk][hk][4 d]), else dq ([n][lq][hq][2 d]).  Rows behind a
// clip's end are zero, whatever their partial results.
template <typename T, bool KEYS>
__global__ __launch_bounds__(256) void attn_sum_kernel(AttnArgs a) {
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int per = (KEYS ? 4 : 2) * a.d / 4, heads = KEYS ? a.hk : a.hq, len = KEYS ? a.lk : a.lq;
  const int64_t rows = static_cast<int64_t>(a.n) * len * heads;
  if (id >= rows * per) return;
  const int64_t row = id / per;
  int col = static_cast<int>(id - row * per) * 4;
  const int head = static_cast<int>(row % heads);
  const int64_t token = row / heads;
  const int clip = static_cast<int>(token / len), at = static_cast<int>(token - static_cast<int64_t>(clip) * len);
  const bool in = at < clip_length(KEYS ? a.k_len : a.q_len, clip, len);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (in) {
    const float *p = a.part + id * 4;
#pragma unroll 4
    for (int i = 0; i < a.splits; ++i) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(p + i * rows * per * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
  }
  struct alignas(4 * sizeof(T)) Four {
    T v[4];
  } x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x.v[e] = static_cast<T>(s[e]);
  T *out;
  if constexpr (KEYS) {
    if (col < 2 * a.d) {
      out = static_cast<T *>(a.dk) + clip * a.dk_batch + at * a.dk_pitch;
      if (!a.dk) return;
    } else {
      out = static_cast<T *>(a.dv) + clip * a.dv_batch + at * a.dv_pitch;
      col -= 2 * a.d;
      if (!a.dv) return;
    }
  } else {
    out = static_cast<T *>(a.dq) + clip * a.dq_batch + at * a.dq_pitch;
  }
  *reinterpret_cast<Four *>(out + static_cast<int64_t>(head) * 2 * a.d + col) = x;
}

__global__ __launch_bounds__(256) void attn_dlam_kernel(AttnArgs a) {
  __shared__ float lds[4];
  sum_dlam(a, blockIdx.x, lds);
}

template <typename T, int D, bool SPLIT>
int launch_dq(AttnArgs a, const BwdPlan &p, hipStream_t s) {
  constexpr int kWaves = kBwdRows / 32;
  using F = Dq<T, D, kWaves>;
  const int e = allow_lds<attn_dq_kernel<T, D, kWaves, SPLIT>>(F::kLds);
  if (e != hipSuccess) return e;
  a.tiles = (a.lq * a.group + kBwdRows - 1) / kBwdRows;
  a.splits = p.dq_splits;
  a.span = p.dq_span;
  a.blocks = static_cast<int64_t>(a.n) * a.hk * a.tiles * a.splits;
  a.part = a.rowstat + p.dq_part;
  if (a.blocks == 0) return hipSuccess;
  attn_dq_kernel<T, D, kWaves, SPLIT><<<grid_of(a.blocks), F::kThreads, F::kLds, s>>>(a);
  if (SPLIT && a.dq) {
    const int64_t threads = static_cast<int64_t>(a.n) * a.lq * a.hq * a.d / 2;
    attn_sum_kernel<T, false><<<static_cast<unsigned>((threads + 255) / 256), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, int D, bool SPLIT, bool DK, bool DV>
int launch_keys(const AttnArgs &a, hipStream_t s) {
  constexpr int kWaves = kBwdRows / 32;
  using F = Dkv<T, D, kWaves>;
  const int e = allow_lds<attn_dkv_kernel<T, D, kWaves, SPLIT, DK, DV>>(F::kLds);
  if (e != hipSuccess) return e;
  static_assert(F::kThreads == 256 && F::kThreads == kBwdThreads, "sum_dlam's workgroup, and what the host checks");
  attn_dkv_kernel<T, D, kWaves, SPLIT, DK, DV><<<grid_of(a.blocks) + a.dlam_blocks, F::kThreads, F::kLds, s>>>(a);
  return hipGetLastError();
}

template <typename T, int D, bool SPLIT>
int launch_dkv(AttnArgs a, const BwdPlan &p, hipStream_t s) {
  a.tiles = (a.lk + kBwdRows - 1) / kBwdRows;
  a.splits = p.dkv_splits;
  a.blocks = static_cast<int64_t>(a.n) * a.hk * a.tiles * a.splits;
  a.part = a.rowstat + p.dkv_part;
  if (a.blocks == 0) return hipSuccess;
  int e = hipSuccess;
  if constexpr (Dkv<T, D, kBwdRows / 32>::kApart) {
    if (a.dk) {
      e = launch_keys<T, D, SPLIT, true, false>(a, s);
      a.dlam_blocks = 0;
    }
    if (e == hipSuccess && a.dv) e = launch_keys<T, D, SPLIT, false, true>(a, s);
  } else {
    e = launch_keys<T, D, SPLIT, true, true>(a, s);
  }
  if (e != hipSuccess) return e;
  if (SPLIT) {
    const int64_t threads = static_cast<int64_t>(a.n) * a.lk * a.hk * a.d;
    attn_sum_kernel<T, true><<<static_cast<unsigned>((threads + 255) / 256), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, int D>
int bwd(const AttnArgs &a, const BwdPlan &p, hipStream_t s) {
  int e = p.dq_splits > 1 ? launch_dq<T, D, true>(a, p, s) : launch_dq<T, D, false>(a, p, s);
  if (e != hipSuccess) return e;
  AttnArgs b = a;
  b.stat_splits = p.dq_splits;
  if ((a.dk || a.dv) && a.n > 0 && a.lk > 0) {
    b.dlam_blocks = a.dlam ? a.hq : 0;
    return p.dkv_splits > 1 ? launch_dkv<T, D, true>(b, p, s) : launch_dkv<T, D, false>(b, p, s);
  }
  if (a.dlam) attn_dlam_kernel<<<a.hq, 256, 0, s>>>(b);
  return hipGetLastError();
}

template <typename T>
int bwd_type(const AttnArgs &a, const BwdPlan &p, hipStream_t s) {
  if (a.d <= 32) return bwd<T, 32>(a, p, s);
  if (a.d <= 64) return bwd<T, 64>(a, p, s);
  return bwd<T, 128>(a, p, s);
}

}  // namespace

int launch_attn_bwd(const AttnArgs &a, const BwdPlan &p, int dtype, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == RT3D_F32) return bwd_type<float>(a, p, s);
  if (dtype == RT3D_BF16) return bwd_type<__bf16>(a, p, s);
  return bwd_type<_Float16>(a, p, s);
}

}  // namespace rt3d
