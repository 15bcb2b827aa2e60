// Device code shared by the kernels of differential attention: MFMA fragments,
// the staged tile and its swizzle, the mask.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>

#include "rt3d_tokens.h"

namespace rt3d {
namespace attn {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) char lds_char;

// A fragment: eight values along the reduction of one row (or column) of a 32x32
// MFMA with 16 reduction steps.  Lane l holds row (column) l % 32, its half h =
// l / 32 the steps 8 h .. 8 h + 7.  For 32-bit values the same eight go through
// eight 32x32x2 products, value e of both halves in the e-th: only the order of
// the sum differs.  Results: lane l holds column l % 32, register i the row
// 8 (i / 4) + 4 h + i % 4.
template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
  using Frag = bf16x8;
  static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<_Float16> {
  using Frag = f16x8;
  static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<float> {
  using Frag = f32x8;
  static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};
template <typename T>
using Frag = typename Mma<T>::Frag;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Waits for this wave's direct loads, then for the workgroup.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Over the two halves of a row (lanes l and l + 32); both get the result.
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Eight consecutive values of a row in memory, 16-byte aligned.
template <typename T>
__device__ __forceinline__ Frag<T> load_frag(const T *p) {
  return *reinterpret_cast<const Frag<T> *>(p);
}
template <>
__device__ __forceinline__ f32x8 load_frag<float>(const float *p) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
  return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// A staged tile: ROWS rows (keys, or query rows) of 2 D values, unpadded (direct
// loads fill LDS in the order of lanes), its 16-byte blocks permuted within
// groups of 16 (8 where a row has only 8) by an XOR with a value of the row.  The
// value makes both kinds of reads free of bank conflicts: 16 rows at one block
// (operands along the row) and four rows at four neighbouring blocks (transposed
// operands).
template <typename T, int D, int ROWS, int THREADS>
struct Tile {
  static constexpr int kEs = sizeof(T);
  static constexpr int kRowBytes = 2 * D * kEs;
  static constexpr int kBlocks = kRowBytes / 16;          // 16-byte blocks of a row
  static constexpr int kBytes = ROWS * kRowBytes;
  static constexpr int kLoads = ROWS * kBlocks / THREADS; // direct loads of a thread
  static_assert(ROWS * kBlocks % THREADS == 0, "a tile is whole loads of every thread");

  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (kBlocks == 8) return ((row & 2) << 1) | ((row >> 2) & 3);
    return ((row & 3) << 2) | ((row >> 2) & 3);
  }

  // A thread's next load lies kStep rows on; where that is a multiple of 16 its
  // block is the same one, and one offset serves for all.
  static constexpr int kStep = THREADS / kBlocks;
  static constexpr int kOffsets = kStep % 16 == 0 ? 1 : kLoads;
  using Offsets = unsigned[kOffsets];

  // Byte offsets of a thread's loads from the tile's first row in memory, or
  // far out of any tile where the block is padding (d < D).  SPLIT: a row is two
  // vectors of d padded to D each (queries, keys), else one of 2 d (values).
  template <bool SPLIT>
  static __device__ __forceinline__ void offsets(int d, int64_t pitch, Offsets &off) {
    constexpr int kPer = 16 / kEs;  // values of a block
#pragma unroll
    for (int i = 0; i < kOffsets; ++i) {
      const int c = i * THREADS + static_cast<int>(threadIdx.x);
      const int row = c / kBlocks, blk = (c % kBlocks) ^ swizzle(row);
      int col = blk * kPer;
      bool in;
      if constexpr (SPLIT) {
        const int m = col / D;
        in = col - m * D < d;
        col = m * d + col - m * D;
      } else {
        in = col < 2 * d;
      }
      off[i] = in ? static_cast<unsigned>((row * pitch + col) * kEs) : 0x80000000u;
    }
  }

  // Starts the loads of `rows` (0..ROWS) rows from `first` on; the other rows
  // of the tile become zeros.
  static __device__ __forceinline__ void stage(const T *first, int rows, int d, int64_t pitch,
                                               const Offsets &off, lds_char *to) {
    const int bytes = rows > 0 ? static_cast<int>(((rows - 1) * pitch + 2 * d) * kEs) : 0;
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(first), 0, bytes, 0x00020000);
    const int wave = uniform(static_cast<int>(threadIdx.x) >> 6);
    const unsigned step = kOffsets == 1 ? static_cast<unsigned>(kStep * pitch * kEs) : 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          r, (__attribute__((address_space(3))) void *)(to + (i * THREADS + wave * 64) * 16), 16,
          static_cast<int>(off[kOffsets == 1 ? 0 : i] + i * step), 0, 0, 0);
  }

  // A lane's address of block 0 of its first row, for both kinds of reads; a
  // block's number only changes bits 4 to 7 of it, by an XOR (tiles begin at
  // multiples of 256 bytes), and rows and blocks beyond those are offsets of the
  // read itself.  `at` adds a tile to it, out of the compiler's sight: it would
  // keep one register for every block otherwise.
  static __device__ __forceinline__ unsigned lane_along() {
    const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
    return row * kRowBytes + (((kEs == 2 ? half : 2 * half) ^ swizzle(row)) << 4);
  }
  static __device__ __forceinline__ unsigned lane_across() {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    if constexpr (kEs == 2) {
      // the transposing read: in 16 lanes, lane 4 r + c reads four values of row
      // r, and receives those of its own column from four rows
      const int row = 4 * half + ((lane & 15) >> 2), sub = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      return row * kRowBytes + ((sub ^ swizzle(row)) << 4) + (lane & 1) * 8;
    } else {
      return 4 * half * kRowBytes + ((((lane & 31) >> 2) ^ half) << 4) + (lane & 3) * 4;
    }
  }
  static __device__ __forceinline__ unsigned at(unsigned lane, const lds_char *tile) {
    unsigned v = lane + static_cast<unsigned>(reinterpret_cast<uintptr_t>(tile));
    asm volatile("" : "+v"(v));
    return v;
  }
  template <typename V>
  static __device__ __forceinline__ V read(unsigned base, int blk, int rows) {
    return *(const __attribute__((address_space(3))) V *)static_cast<uintptr_t>(
        (base ^ ((blk & 15) << 4)) + (blk & ~15) * 16 + rows * kRowBytes);
  }

  // Operand along the row: eight values from column `col` + 8 half of row row0 +
  // lane % 32 (row0, col: constants, multiples of 32 and 16).
  static __device__ __forceinline__ Frag<T> along(unsigned base, int row0, int col) {
    if constexpr (kEs == 2) return read<Frag<T>>(base, col / 8, row0);
    const auto a = read<f32x4>(base, col / 4, row0), b = read<f32x4>(base, col / 4 + 1, row0);
    return Frag<T>{static_cast<T>(a[0]), static_cast<T>(a[1]), static_cast<T>(a[2]), static_cast<T>(a[3]),
                   static_cast<T>(b[0]), static_cast<T>(b[1]), static_cast<T>(b[2]), static_cast<T>(b[3])};
  }

  // Transposed operand: column `col` + lane % 32, and of the 16 rows from row0
  // on those that a result's registers hold for the half: value e is row
  // row0 + 8 (e / 4) + 4 half + e % 4.  row0 and col: multiples of 16 and 32.
  static __device__ __forceinline__ Frag<T> across(unsigned base, int row0, int col) {
    if constexpr (kEs == 2) {
      union {
        s16x4 half4[2];
        Frag<T> all;
      } u;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int blk = (col / 8) ^ (2 * j);  // rows 8 further on: their swizzle differs by 2
        u.half4[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)static_cast<uintptr_t>(
                (base ^ ((blk & 15) << 4)) + (blk & ~15) * 16 + (row0 + 8 * j) * kRowBytes));
      }
      return u.all;
    } else {
      Frag<T> v;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = read<T>(base, (col / 4) ^ ((e % 4) << 2 | 2 * (e / 4)), row0 + 8 * (e / 4) + e % 4);
      return v;
    }
  }
};

// Eight result registers as an operand whose reduction runs over their rows (the
// order that `across` reads the other operand in); rounded to the layer's type.
template <typename T>
__device__ __forceinline__ Frag<T> pack(const f32x16 &v, int from) {
  Frag<T> f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = static_cast<T>(v[from + e]);
  return f;
}

// acc += a chain of N products whose first operands, read(i), come from LDS up to
// four products ahead of their use; second(i) is at hand.  (Left to itself the
// compiler reads, waits and multiplies.  dk/dv has no registers for it at d = 64: there it
// spilled and cost 3%.)
template <typename T, int N, typename R, typename S>
__device__ __forceinline__ f32x16 chain(R read, S second, f32x16 acc) {
  constexpr int kRing = N < 4 ? N : 4;
  Frag<T> f[kRing];
#pragma unroll
  for (int i = 0; i < kRing; ++i) f[i] = read(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    acc = Mma<T>::run(f[i % kRing], second(i), acc);
    if (i + kRing < N) f[i % kRing] = read(i + kRing);
    __builtin_amdgcn_sched_barrier(0);
  }
  return acc;
}

// The same with both operands in LDS.
template <typename T, int N, typename R, typename S>
__device__ __forceinline__ f32x16 chain_both(R read, S second, f32x16 acc) {
  constexpr int kRing = N < 4 ? N : 4;
  Frag<T> f[kRing], g[kRing];
#pragma unroll
  for (int i = 0; i < kRing; ++i) f[i] = read(i), g[i] = second(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    acc = Mma<T>::run(f[i % kRing], g[i % kRing], acc);
    if (i + kRing < N) f[i % kRing] = read(i + kRing), g[i % kRing] = second(i + kRing);
    __builtin_amdgcn_sched_barrier(0);
  }
  return acc;
}

// Row of a result register.
__device__ __forceinline__ int result_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// Keys visible to query i of a clip: the first `visible` ones.  The queries end
// where the keys end; with frames, a query sees its own frame and those before.
__device__ __forceinline__ int visible(int i, int q_len, int k_len, int frame) {
  if (!frame) return k_len;
  const int p = k_len - q_len + i;
  if (p < 0) return 0;
  const int64_t end = (static_cast<int64_t>(p / frame) + 1) * frame;
  return end < k_len ? static_cast<int>(end) : k_len;
}

__device__ __forceinline__ int clip_length(const int32_t *len, int clip, int most) {
  if (!len) return most;
  const int v = len[clip];
  return v < 0 ? 0 : v > most ? most : v;
}

// What a workgroup does: tile number `rank` of those of a pair (clip, key head), in
// the order of their work, and which split of it.
struct Place {
  int split, rank, kvh, clip;
};

// Workgroups of a pair read the same keys (or queries).  Without a causal mask they
// follow one another on one XCD (ids go round the eight), whose L2 then serves them;
// or, where clips of unlike lengths would leave XCDs with unlike work, on all.  With
// one, the tiles with most work of all pairs come first, so that the last ones to
// start are short: the pairs are dealt to the XCDs in as many sets as divide both.
// (4 clips of 4096 tokens, 8 heads, d 64, forward and backward: 811 us, pair after
// pair 1014; one clip of 3 heads, whose sets no number of XCDs shares, 209 and 203.)
// walk: the clips' walks where they differ (NULL: all `most`).  Up to 64 clips, a lane
// each, the longest come first: 6 random ones up to 3136 tokens 482 us, 517 in the
// order of the batch; 3 up to 4096 662 and 657.
// False: the workgroup has no work.
__device__ __forceinline__ bool place(const AttnArgs &a, const int32_t *walk, int most, Place &p) {
  unsigned id = blockIdx.x;
  if (!a.sets && !a.spread) {
    const unsigned per = static_cast<unsigned>(a.blocks + 7) / 8;  // blocks < 2^31
    id = (id % 8) * per + id / 8;
  }
  if (id >= a.blocks) return false;
  const unsigned splits = a.splits, tiles = a.tiles;
  unsigned pair;
  if (a.sets) {
    const unsigned sets = a.sets, pairs = static_cast<unsigned>(a.n) * a.hk / sets, set = id % sets;
    id /= sets;
    const unsigned split = id % splits;
    id /= splits;
    p.rank = static_cast<int>(id / pairs);
    pair = set * pairs + id % pairs;
    // A causal split has more work the earlier it is: the splits of neighbouring tiles
    // change places, or those of one kind would meet on the same XCDs and CUs.  (8000
    // tokens, 4 heads, d 64, two splits: forward 159 us, 175 without.)
    p.split = static_cast<int>((split + __builtin_popcount(p.rank)) % splits);
  } else {
    p.split = static_cast<int>(id % splits);
    id /= splits;
    p.rank = static_cast<int>(id % tiles);
    pair = id / tiles;
  }
  p.clip = static_cast<int>(pair / a.hk);
  p.kvh = static_cast<int>(pair - static_cast<unsigned>(p.clip) * a.hk);
  if (!a.sets && walk && a.n <= 64) {
    // clip number p.clip of those in the order of their walks
    const int lane = threadIdx.x & 63, mine = lane < a.n ? clip_length(walk, lane, most) : -1;
    int before = 0;
    for (int i = 0; i < a.n; ++i) {
      const int other = __builtin_amdgcn_readlane(mine, i);
      before += other > mine || (other == mine && i < lane);
    }
    p.clip = uniform(__builtin_ctzll(__ballot(lane < a.n && before == p.clip)));
  }
  return true;
}
inline unsigned grid_of(int64_t blocks) { return static_cast<unsigned>((blocks + 7) / 8 * 8); }

// Lets a kernel use more than the default 64 KB of LDS, once per device.
template <auto K>
int allow_lds(int bytes) {
  if (bytes <= 65536) return hipSuccess;
  constexpr int kMost = 64;
  static std::atomic<bool> done[kMost];
  int dev = 0;
  const hipError_t got = hipGetDevice(&dev);
  if (got != hipSuccess) return got;
  const bool known = dev >= 0 && dev < kMost;
  if (known && done[dev].load(std::memory_order_acquire)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(K),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess && known) done[dev].store(true, std::memory_order_release);
  return e;
}

}  // namespace attn
}  // namespace rt3d
