// Attention of one new token of each sequence over a paged key-value cache,
// split over the cache's length and joined:
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),
// j over the sequence's tokens (the last `window` of them), m a running
// maximum; o = 0 and lse = -inf where there is none, or no score above -inf.
//
// Bound by the cache's bytes: each key and value is read once, straight into
// registers in the layout the matrix cores take, and serves all query heads
// that share it (up to 16 a wave; more come in further blocks).  A wave works
// on 32 tokens at a time:
//   S^T = K Q^T   rows are tokens, columns heads.  Lane group g (lane / 16)
//                 holds scores of tokens 4 g + 0..3 and 16 + 4 g + 0..3, which
//                 is the order in which it then gives p to
//   O^T = V^T P^T whose sum over tokens may run in any order.  Lane c of a
//                 group loads the same contiguous dims of the group's eight
//                 tokens; the operand's pairs (two tokens, one dim) are byte
//                 permutations of its own registers, so V needs no LDS.
// The running maximum moves only when a score passes it by more than 2^8 (2^4
// with float16), so that the usual tile needs no exchange between lanes and no
// rescaling.  p is handed over in parts of T that add up to it: three of
// bfloat16 are all of its 24 bits; two of float16 are 22, with p 2^11 times as
// large, so that what falls below its smallest value is under 2^-36 of the
// largest p.  Sums and statistics are float32.
//
// Caches of 4 bits are e2m1 codes with a power of two for each 32 dims: an
// instruction widens two codes and applies the power, exactly (past T's range: infinite).  16
// sequences of 65536 tokens of 4 heads of 128 in 113 us (4.8 TB/s); 24 of 28000 of 16 heads of 64 in
// 177 us with the join (4.1 TB/s).  On shorter ones, 24 of 6900 in 54 us (3.3 TB/s), start and end weigh
// more, and where lengths differ (24 of up to 6900: 30 us and 5 for the join) runs cut by the longest leave
// half of the blocks without tokens; two tiles that share the columns of one softmax where query heads
// are few (a tenth fewer vector instructions) changed nothing.
//
// MASS: the kernel also leaves its scores, and what each token's weights come to
// is added to its mass once the sums of all runs are known: by the same block
// where it has all of them, else beside the join (131072 tokens of 28 heads on 4:
// 7.8 us with the join, which is 5 alone).
#pragma once

#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// What a cache holds: the queries' type, e4m3 with a scale a head, e2m1 with block exponents.
enum class Held { kSame, kE4m3, kE2m1 };

constexpr int kTile = 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// In powers of two: how far a score may pass the running maximum, and the
// largest p until one does.  Their sum stays inside T's range, and with bfloat16
// no p passes 1, so that values near the ends of its range stay inside float32.
template <class T> constexpr float kSlack = 8.f;
template <class T> constexpr float kLift = -8.f;
template <> constexpr float kSlack<F16> = 4.f;
template <> constexpr float kLift<F16> = 11.f;

// 32 x 16 pieces of a head's dims held by a lane of the value operand: runs of
// 8, 4 and 2 dims, from 128, 64 and 32 dims of the head.
template <int D>
struct Dims {
  static constexpr int n8 = D / 128, n4 = D % 128 / 64, n2 = D % 64 / 32;
  static constexpr int pairs = D / 32;          // packed pairs a lane holds of a token
};

// A lane's dims of one token's value row, as they are stored, and as packed pairs of T.
template <class T, Held C, int D>
struct RawValue {
  using L = Dims<D>;
  static constexpr bool C8 = C == Held::kE4m3;
  static constexpr int kWords = C8 ? (L::pairs + 1) / 2 : L::pairs;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const uint8_t* row, const uint8_t*, int c) {
    constexpr int kB = C8 ? 1 : 2;
#pragma unroll
    for (int i = 0; i < L::n8; ++i) {
      if constexpr (C8) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(row + i * 128 + c * 8);
        w[2 * i] = v[0];
        w[2 * i + 1] = v[1];
      } else {
        const u32x4 v = *reinterpret_cast<const u32x4*>(row + i * 256 + c * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
      }
    }
    const uint8_t* rest = row + L::n8 * 128 * kB;
    constexpr int at = L::n8 * (C8 ? 2 : 4);
    if constexpr (L::n4) {
      if constexpr (C8) {
        w[at] = *reinterpret_cast<const uint32_t*>(rest + c * 4);
      } else {
        const u32x2 v = *reinterpret_cast<const u32x2*>(rest + c * 8);
        w[at] = v[0];
        w[at + 1] = v[1];
      }
    }
    if constexpr (L::n2) {
      const uint8_t* last = rest + L::n4 * 64 * kB;
      if constexpr (C8) w[at + L::n4] = *reinterpret_cast<const uint16_t*>(last + c * 2);
      else w[at + 2 * L::n4] = *reinterpret_cast<const uint32_t*>(last + c * 4);
    }
  }
  // Packed pair q.
  __device__ __forceinline__ uint32_t pair(int q) const {
    if constexpr (!C8) return w[q];
    return q % 2 == 0 ? widen2<T, false>(w[q / 2]) : widen2<T, true>(w[q / 2]);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
};

// Of a 4-bit cache: a word, half a word and a byte of codes for the runs of 8, 4 and 2
// dims, and the exponent byte of the block that each run lies in.
template <class T, int D>
struct RawValue<T, Held::kE2m1, D> {
  using L = Dims<D>;
  static constexpr int kRuns = L::n8 + L::n4 + L::n2;
  uint32_t w[kRuns], e[kRuns];

  __device__ __forceinline__ void load(const uint8_t* row, const uint8_t* exps, int c) {
#pragma unroll
    for (int i = 0; i < L::n8; ++i) {
      w[i] = *reinterpret_cast<const uint32_t*>(row + i * 64 + c * 4);
      e[i] = exps[i * 4 + c / 4];
    }
    if constexpr (L::n4) {
      w[L::n8] = *reinterpret_cast<const uint16_t*>(row + L::n8 * 64 + c * 2);
      e[L::n8] = exps[L::n8 * 4 + c / 8];
    }
    if constexpr (L::n2) {
      w[L::n8 + L::n4] = row[L::n8 * 64 + L::n4 * 32 + c];
      e[L::n8 + L::n4] = exps[L::n8 * 4 + L::n4 * 2];
    }
  }
  __device__ __forceinline__ uint32_t pair(int q) const {
    const int run = q < 4 * L::n8 ? q / 4 : q < 4 * L::n8 + 2 * L::n4 ? L::n8 : L::n8 + L::n4;
    const int byte = q < 4 * L::n8 ? q % 4 : q < 4 * L::n8 + 2 * L::n4 ? q - 4 * L::n8 : 0;
    return open2<T>(w[run], power_of(e[run]), byte);
  }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t most = e[0];
#pragma unroll
    for (int i = 1; i < kRuns; ++i) most = max(most, e[i]);
    return most;
  }
  // Codes and exponent both, so that a block without a value (exponent 255) counts nothing.
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kRuns; ++i) w[i] = e[i] = 0;
  }
};

// The dims of step j that lane group g takes of a key and of the query, and
// how a key's are loaded: eight at a time (16 bytes), or with 8-bit caches
// sixteen, for two steps, and with 4-bit ones a quarter of the row.
template <Held C, int D>
__device__ __forceinline__ int key_dim(int j, int g) {
  if (C == Held::kE2m1) return g * (D / 4) + j * 8;
  if (C == Held::kE4m3 && j / 2 * 64 + 64 <= D) return j / 2 * 64 + g * 16 + j % 2 * 8;
  return j * 32 + g * 8;
}
template <class T, Held C, int D>
struct RawKey {
  static constexpr bool C8 = C == Held::kE4m3;
  static constexpr int kSteps = D / 32;
  u32x4 w[C8 ? (kSteps + 1) / 2 : kSteps];

  // row: the token's row, past the lane group's first dims (16 g bytes, or 8 g
  // where the last step is alone).
  __device__ __forceinline__ void load(const uint8_t* row, const uint8_t*, int g) {
    if constexpr (!C8) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) w[j] = *reinterpret_cast<const u32x4*>(row + j * 64 + g * 16);
    } else {
#pragma unroll
      for (int j = 0; j < kSteps / 2; ++j) w[j] = *reinterpret_cast<const u32x4*>(row + j * 64 + g * 16);
      if constexpr (kSteps % 2) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(row + kSteps / 2 * 64 + g * 8);
        w[kSteps / 2][0] = v[0];
        w[kSteps / 2][1] = v[1];
      }
    }
  }
  __device__ __forceinline__ u32x4 step(int j, int) const {
    if constexpr (!C8) return w[j];
    const uint32_t a = w[j / 2][j % 2 * 2], b = w[j / 2][j % 2 * 2 + 1];
    return u32x4{widen2<T, false>(a), widen2<T, true>(a), widen2<T, false>(b), widen2<T, true>(b)};
  }
};

// Of a 4-bit cache: a word of codes for each step, and the exponents of the blocks that
// the lane group's quarter of the row begins and ends in.
template <class T, int D>
struct RawKey<T, Held::kE2m1, D> {
  static constexpr int kSteps = D / 32, kQuarter = D / 4;
  static constexpr bool kTwo = kQuarter > 32 || 32 % kQuarter != 0;
  uint32_t w[kSteps], e[2];

  __device__ __forceinline__ void load(const uint8_t* row, const uint8_t* exps, int g) {
    const uint8_t* at = row + g * (kQuarter / 2);
    if constexpr (kSteps % 4 == 0) {
#pragma unroll
      for (int j = 0; j < kSteps; j += 4) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(at + j * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[j + i] = v[i];
      }
    } else if constexpr (kSteps % 2 == 0) {
#pragma unroll
      for (int j = 0; j < kSteps; j += 2) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(at + j * 4);
        w[j] = v[0];
        w[j + 1] = v[1];
      }
    } else {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) w[j] = *reinterpret_cast<const uint32_t*>(at + j * 4);
    }
    e[0] = exps[g * kQuarter / 32];
    if constexpr (kTwo) e[1] = exps[(g * kQuarter + kQuarter - 8) / 32];
  }
  __device__ __forceinline__ u32x4 step(int j, int g) const {
    const bool second = kTwo && (g * kQuarter + j * 8) / 32 != g * kQuarter / 32;
    const float s = power_of(second ? e[1] : e[0]);
    return u32x4{open2<T>(w[j], s, 0), open2<T>(w[j], s, 1), open2<T>(w[j], s, 2), open2<T>(w[j], s, 3)};
  }
};

// Two p as packed pairs of T that add up to them, the largest part first.  An
// infinite value has to meet no part of another sign and, while p is not 0, no
// part of 0: bfloat16's parts are cut below what they are parts of, so that
// there is always a rest (p from 2^-90 on), and a float16 p's rest meets the
// values through finite2.
// (Over 4 bits two parts of bfloat16, 2^-17 of p, took 4 % less, 111 against 115 us for
// 16 x 65536 tokens, and put two to ten times as many results a step of bfloat16 off.)
template <class T> constexpr int kParts = 3;
template <> constexpr int kParts<F16> = 2;
template <class T>
__device__ __forceinline__ void split(float a, float b, uint32_t* part);
template <>
__device__ __forceinline__ void split<Bf16>(float a, float b, uint32_t* part) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // The float below, or 0.
    const uint32_t x = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u), y = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u);
    part[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    a -= __uint_as_float(x & 0xffff0000u);
    b -= __uint_as_float(y & 0xffff0000u);
  }
  part[2] = pack2<Bf16>(a, b);
}
template <>
__device__ __forceinline__ void split<F16>(float a, float b, uint32_t* part) {
  part[0] = pack2<F16>(a, b);
  const float2 r = unpack2<F16>(part[0]);
  part[1] = pack2<F16>(a - r.x, b - r.y);
}
// A packed pair of float16 with infinities as the largest numbers.  (NaN may
// become one too; the largest part of p meets the pair as it is.)
__device__ __forceinline__ uint32_t finite2(uint32_t w) {
  const f16x2 most = {(_Float16)65504.f, (_Float16)65504.f};
  const f16x2 v = __builtin_elementwise_max(__builtin_elementwise_min(__builtin_bit_cast(f16x2, w), most), -most);
  return __builtin_bit_cast(uint32_t, v);
}

// Loads above stay above: the compiler would move a load that the next turn of
// a loop uses to where it uses it.
__device__ __forceinline__ void keep_loads_here() { asm volatile("" ::: "memory"); }

// One (sequence, key-value head, up to 16 of its query heads, run of tiles).
// Partial results of run s: o [head][D], then m and l, unnormalised.
// UNI: pages are multiples of a tile, so a tile's tokens follow each other in
// memory and its address is the wave's; otherwise each lane finds one token's
// row and the lanes exchange them.
template <class T, Held C, int D, int W, bool UNI, bool MASS>
__global__ __launch_bounds__(64 * W, W == 16 ? 1 : 2) void attend_kernel(AttendParams p, int tiles_per_run, int runs, float* part_o,
                                                           float* part_ml, float* scores, bool whole) {
  extern __shared__ __attribute__((aligned(16))) float s_x[];   // MASS, whole: the scores [heads][tokens]
  constexpr int kSteps = D / 32;
  using L = Dims<D>;
  __shared__ float s_o[W][16][D + 4];
  __shared__ float s_m[W][16], s_l[W][16];
  __shared__ float s_top[MASS ? 16 : 1], s_sum[MASS ? 16 : 1];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane % 16, g = lane / 16;
  const int group = p.hq / p.hk, head_tiles = (group + 15) / 16;
  const int run = blockIdx.x, kh = blockIdx.y / head_tiles, h0 = kh * group + blockIdx.y % head_tiles * 16;
  const int heads = min(16, (kh + 1) * group - h0);
  const int b = blockIdx.z;
  if (run >= runs) return;

  const int hi = max(0, int(min(int64_t(__builtin_amdgcn_readfirstlane(p.lengths[b])), p.max_length)));
  const int lo = p.window > 0 ? max(0, hi - p.window) : 0;
  const int tile0 = lo / kTile + run * tiles_per_run;
  const int tile1 = min((hi + kTile - 1) / kTile, tile0 + tiles_per_run);
  const int32_t* table = p.table + int64_t(b) * p.width;
  constexpr int kRow = C == Held::kSame ? D * 2 : C == Held::kE4m3 ? D : D / 2;
  constexpr int kExps = C == Held::kE2m1 ? D / 32 : 0;
  const uint8_t* kc = static_cast<const uint8_t*>(p.k_cache);
  const uint8_t* vc = static_cast<const uint8_t*>(p.v_cache);

  u32x4 q[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    q[j] = u32x4{0, 0, 0, 0};
    if (c < heads)
      q[j] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.q) + (int64_t(b) * p.hq + h0 + c) * D + key_dim<C, D>(j, g));
  }
  const float to_log2 = p.scale * kLog2e * (p.k_scale ? p.k_scale[kh] : 1.f);

  // m: log2 of the score whose p is 1, kLift below the running maximum.
  float m = -INFINITY, l = 0.f;
  f32x4 o[2 * L::pairs];
#pragma unroll
  for (int i = 0; i < 2 * L::pairs; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Which token of a tile this lane looks up: one each, or the tile's first.
  // Tokens outside [lo, hi) take the nearest one inside (their p is 0).
  auto token = [&](int tile) { return UNI ? tile * kTile : min(max(tile * kTile + lane % 32, lo), hi - 1); };
  auto page_index = [&](int t) { return int(__umulhi(2u * unsigned(t), p.page_magic) >> p.page_shift); };
  auto look_up = [&](int tile) { return table[page_index(token(min(tile, tile1 - 1)))]; };
  auto row_of = [&](int tile, int32_t entry) {
    const int t = token(tile);
    const unsigned page = min(unsigned(UNI ? __builtin_amdgcn_readfirstlane(entry) : entry), unsigned(p.pages - 1));
    return (page * unsigned(p.hk) + unsigned(kh)) * unsigned(p.page) + unsigned(t - page_index(t) * p.page);
  };
  // Row of the tile's token i, where lanes of a group want different ones, and the bytes before it: a wave's
  // base and a small offset (e4m3 of 64 and 128 dims 92 and 116 registers, with the row times the bytes 117 and 146; 16
  // sequences of 8192 tokens of 256 dims in bfloat16 126 us against 140).  Where codes and exponents are both read
  // it is the row, found once (float16 queries of 64 and 128 dims 114 and 145 registers, 131 and 160 otherwise).
  auto row = [&](unsigned mine, int i) { return UNI ? uint64_t(mine) + unsigned(i) : uint64_t(unsigned(__shfl(int(mine), i))); };
  auto bytes = [&](unsigned mine, int i) { return UNI ? uint64_t(mine) * kRow + unsigned(i) * kRow : row(mine, i) * kRow; };
  RawKey<T, C, D> key[2];
  RawValue<T, C, D> val[8];
  auto load = [&](auto& to, const uint8_t* cache, const uint8_t* exps, unsigned mine, int i, int of) {
    if constexpr (C == Held::kE2m1) {
      const uint64_t r = row(mine, i);
      to.load(cache + r * kRow, exps + r * kExps, of);
    } else {
      to.load(cache + bytes(mine, i), nullptr, of);
    }
  };
  auto load_keys = [&](unsigned mine) {
#pragma unroll
    for (int i = 0; i < 2; ++i) load(key[i], kc, p.k_exps, mine, i * 16 + c, g);
    keep_loads_here();
  };
  auto load_values = [&](unsigned mine) {
#pragma unroll
    for (int i = 0; i < 8; ++i) load(val[i], vc, p.v_exps, mine, i / 4 * 16 + g * 4 + i % 4, c);
    keep_loads_here();
  };

  // One tile.  The next one's keys are loaded as soon as this one's are used,
  // its values likewise, the page of the one after that meanwhile: a wave has
  // a tile under way all the time without a second set of registers.
  int32_t entry = 0;
  auto work = [&](auto more, int tile) {
    const int t0 = tile * kTile;
    f32x4 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kSteps; ++j) s[i] = mfma32<T>(key[i].step(j, g), q[j], s[i]);
    }
    unsigned next = 0;
    if (more) {
      next = row_of(tile + W, entry);
      load_keys(next);
      entry = look_up(tile + 2 * W);
      keep_loads_here();
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[i / 4][i % 4] * to_log2;
    if (t0 < lo || t0 + kTile > hi) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = t0 + i / 4 * 16 + g * 4 + i % 4;
        if (at < lo || at >= hi) {
          x[i] = -INFINITY;
          val[i].clear();
        }
      }
    }
    if constexpr (MASS) {
      if (c < heads) {
        const int64_t stride = int64_t(runs) * tiles_per_run * kTile;
        float* to = (whole ? s_x + c * stride : scores + (int64_t(b) * p.hq + h0 + c) * stride) + int64_t(tile - lo / kTile) * kTile + g * 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4*>(to + i * 16) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
    if (__any(top > m + (kSlack<T> + kLift<T>))) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m2 = fmaxf(m, top - kLift<T>);
      const float f = m2 == m ? 1.f : __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int i = 0; i < 2 * L::pairs; ++i) o[i] *= f;
    }
    // While no score is above -inf, each p is 0.
    const float base = m == -INFINITY ? 0.f : m;
    constexpr int kOf = kParts<T>;
    u32x4 part[kOf];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float a = __builtin_amdgcn_exp2f(x[i] - base), e = __builtin_amdgcn_exp2f(x[i + 1] - base);
      l += a + e;
      uint32_t w[kOf];
      split<T>(a, e, w);
#pragma unroll
      for (int n = 0; n < kOf; ++n) part[n][i / 2] = w[n];
    }
    // Whether values may be infinite in float16.  6 times 2^13 is not, and 4-bit blocks past that are rare,
    // so they are looked for (24 sequences of up to 6900 tokens 33.8 us; 38.5 with finite2 for all, 32.5 with neither).
    bool past = std::is_same_v<T, F16> && C == Held::kSame;
    if constexpr (std::is_same_v<T, F16> && C == Held::kE2m1) {
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = max(most, val[j].largest());
      past = __any(most > 127 + 13);
    }
#pragma unroll
    for (int i = 0; i < L::pairs; ++i) {
      u32x4 even, odd;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t a = val[2 * j].pair(i), e = val[2 * j + 1].pair(i);
        even[j] = __builtin_amdgcn_perm(e, a, 0x05040100u);
        odd[j] = __builtin_amdgcn_perm(e, a, 0x07060302u);
      }
#pragma unroll
      for (int n = 0; n < kOf; ++n) {
        if (std::is_same_v<T, F16> && C != Held::kE4m3 && n == 1 && past) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            even[j] = finite2(even[j]);
            odd[j] = finite2(odd[j]);
          }
        }
        o[2 * i] = mfma32<T>(even, part[n], o[2 * i]);
        o[2 * i + 1] = mfma32<T>(odd, part[n], o[2 * i + 1]);
      }
    }
    if (more) load_values(next);
  };
  int tile = tile0 + wave;
  if (tile < tile1) {
    const unsigned first = row_of(tile, look_up(tile));
    // In the order of the loop, so that its waits are for just what they need.
    load_keys(first);
    entry = look_up(tile + W);
    keep_loads_here();
    load_values(first);
    for (; tile + W < tile1; tile += W) work(std::true_type(), tile);
    work(std::false_type(), tile);
  }

  // The block's waves meet.  o[2 i + e] of lane (g, c): head c, dims of the
  // operand's rows 4 g + 0..3, that is of lanes 4 g + 0..3, pair i, element e.
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    s_m[wave][c] = m;
    s_l[wave][c] = l;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float* row = s_o[wave][c];
    const int cc = g * 4 + r;
#pragma unroll
    for (int i = 0; i < L::n8; ++i)
#pragma unroll
      for (int e = 0; e < 8; e += 4)
        *reinterpret_cast<f32x4*>(row + i * 128 + cc * 8 + e) =
            f32x4{o[8 * i + e][r], o[8 * i + e + 1][r], o[8 * i + e + 2][r], o[8 * i + e + 3][r]};
    constexpr int at = 8 * L::n8;
    if constexpr (L::n4)
      *reinterpret_cast<f32x4*>(row + L::n8 * 128 + cc * 4) = f32x4{o[at][r], o[at + 1][r], o[at + 2][r], o[at + 3][r]};
    if constexpr (L::n2)
      *reinterpret_cast<f32x2*>(row + L::n8 * 128 + L::n4 * 64 + cc * 2) = f32x2{o[at + 4 * L::n4][r], o[at + 4 * L::n4 + 1][r]};
  }
  __syncthreads();
  const float vs = p.v_scale ? p.v_scale[kh] : 1.f;
  // The token whose mass this thread adds to, in a block that has all of its key-value head.
  int t = lo + int(threadIdx.x);
  float* mass = MASS ? p.mass + (int64_t(b) * p.hk + kh) * p.mass_span : nullptr;
  float before = MASS && whole && t < hi ? mass[t] : 0.f;
  for (int i = threadIdx.x; i < heads * (D / 4); i += 64 * W) {
    const int h = i / (D / 4), d = i % (D / 4) * 4;
    float M = s_m[0][h];
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, s_m[w][h]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (s_l[w][h] == 0.f) continue;         // a wave without tokens
      const float f = __builtin_amdgcn_exp2f(s_m[w][h] - M);
      acc += *reinterpret_cast<const f32x4*>(&s_o[w][h][d]) * f;
      sum = fmaf(s_l[w][h], f, sum);
    }
    const int64_t row = int64_t(b) * p.hq + h0 + h;
    if (whole) {
      const float k = vs / sum;
      u32x2 v;
#pragma unroll
      for (int e = 0; e < 2; ++e) v[e] = sum == 0.f ? 0u : pack2<T>(acc[2 * e] * k, acc[2 * e + 1] * k);
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + row * D + d) = v;
      if (p.lse && d == 0) p.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
      if (MASS && d == 0) {
        s_top[h] = M;
        s_sum[h] = sum;
      }
    } else {
      *reinterpret_cast<f32x4*>(part_o + (row * runs + run) * D + d) = acc;
      if (d == 0) *reinterpret_cast<f32x2*>(part_ml + (row * runs + run) * 2) = f32x2{M, sum};
    }
  }
  if (!MASS || !whole) return;
  lds_sync();
  for (; t < hi; t += 64 * W) {
    const float* x = s_x + (t - lo / kTile * kTile);
    float more = 0.f;
#pragma unroll 4
    for (int h = 0; h < heads; ++h)
      if (s_sum[h] != 0.f) more = fmaf(__builtin_amdgcn_exp2f(x[h * tiles_per_run * kTile] - s_top[h]), 1.f / s_sum[h], more);
    mass[t] = before + more;
    before = t + 64 * W < hi ? mass[t + 64 * W] : 0.f;
  }
}

// mass[b, kh, t] += sum over the heads of kh of p_t / sum_j p_j, two tokens a thread:
// block `id` has 2 THREADS consecutive ones of a (sequence, key-value head).  Its waves
// find sixteen heads' maxima and sums from those of their runs, while the scores are on
// their way, then all add up the heads.
template <int THREADS>
__device__ __forceinline__ void add_mass(const AttendParams& p, int64_t id, int runs, const float* part_ml, const float* scores,
                                         int64_t stride) {
  __shared__ float s_top[16], s_rec[16];
  const int64_t chunks = (stride + 2 * THREADS - 1) / (2 * THREADS), bk = id / chunks;
  if (bk >= int64_t(p.batch) * p.hk) return;
  const int64_t b = bk / p.hk, at = (id - bk * chunks) * (2 * THREADS) + threadIdx.x;
  const int kh = int(bk - b * p.hk), group = p.hq / p.hk, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int hi = max(0, int(min(int64_t(p.lengths[b]), p.max_length)));
  const int lo = p.window > 0 ? max(0, hi - p.window) : 0;
  const int64_t t = lo / kTile * kTile + at;
  if (t - int(threadIdx.x) >= hi) return;
  const int64_t row0 = b * p.hq + int64_t(kh) * group;
  float* mass = p.mass + bk * p.mass_span + t;
  bool here[2];
  float before[2], more[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    here[i] = t + i * THREADS >= lo && t + i * THREADS < hi;
    before[i] = here[i] ? mass[i * THREADS] : 0.f;
  }
  for (int h0 = 0; h0 < group; h0 += 16) {
    const int heads = min(16, group - h0);
    float x[2][16];
#pragma unroll
    for (int h = 0; h < 16; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) x[i][h] = h < heads && here[i] ? scores[(row0 + h0 + h) * stride + at + i * THREADS] : 0.f;
    for (int h = wave; h < heads; h += THREADS / kWave) {
      const float2* ml = reinterpret_cast<const float2*>(part_ml) + (row0 + h0 + h) * runs;
      float M = -INFINITY, sum = 0.f;
#pragma unroll 4
      for (int s = lane; s < runs; s += kWave) {
        const float2 v = ml[s];
        if (v.y == 0.f) continue;
        const float top = fmaxf(M, v.x);
        sum = fmaf(v.y, __builtin_amdgcn_exp2f(v.x - top), sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f(M - top));
        M = top;
      }
      const float top = wave_max(M);
      sum = wave_sum(sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f(M - top));
      if (lane == 0) {
        s_top[h] = top;
        s_rec[h] = sum == 0.f ? 0.f : 1.f / sum;      // 0: no score above -inf
      }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 16; ++h)
      if (h < heads && s_rec[h] != 0.f)
#pragma unroll
        for (int i = 0; i < 2; ++i) more[i] = fmaf(__builtin_amdgcn_exp2f(x[i][h] - s_top[h]), s_rec[h], more[i]);
    if (h0 + 16 < group) __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (here[i]) mass[i * THREADS] = before[i] + more[i];
}

// The runs of one (sequence, query head) joined, DIMS dims a block.  The runs'
// weights are found once, in LDS; then DIMS / 4 threads read their part of a
// run and the block's other threads those of others, four runs under way each.
template <class T, int DIMS, int kJoinThreads, bool MASS>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendParams p, int runs, const float* part_o,
                                                                   const float* part_ml, const float* scores, int64_t stride) {
  constexpr int kLanes = DIMS / 4, kRows = kJoinThreads / kLanes, kWaves = kJoinThreads / kWave;
  extern __shared__ float s_f[];                // [runs] weights
  __shared__ float s_red[2][kWaves];
  __shared__ f32x4 s_acc[kRows][kLanes];
  if constexpr (MASS) {
    const int64_t rows = int64_t(p.batch) * p.hq;
    if (blockIdx.x >= rows) {
      add_mass<kJoinThreads>(p, (blockIdx.x - rows) * gridDim.y + blockIdx.y, runs, part_ml, scores, stride);
      return;
    }
  }
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, wave = tid / kWave, r = tid / kLanes, c = tid % kLanes;
  const float2* ml = reinterpret_cast<const float2*>(part_ml) + row * runs;
  const f32x4* o = reinterpret_cast<const f32x4*>(part_o + row * runs * p.d + blockIdx.y * DIMS) + c;
  const int step = p.d / 4;
  // The first rows and statistics are on their way together.
  f32x4 early[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) early[x] = o[int64_t(min(r + x * kRows, runs - 1)) * step];
  const float2 mine = ml[min(tid, runs - 1)];
  float M = mine.y != 0.f ? mine.x : -INFINITY;
  for (int s = tid + kJoinThreads; s < runs; s += kJoinThreads) {
    const float2 v = ml[s];
    if (v.y != 0.f) M = fmaxf(M, v.x);
  }
  M = wave_max(M);
  if (tid % kWave == 0) s_red[0][wave] = M;
  __syncthreads();
  M = s_red[0][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_red[0][w]);
  float sum = 0.f;
  for (int s = tid; s < runs; s += kJoinThreads) {
    const float2 v = s == tid ? mine : ml[s];
    const float f = v.y != 0.f ? __builtin_amdgcn_exp2f(v.x - M) : 0.f;
    s_f[s] = f;
    sum = v.y != 0.f ? fmaf(v.y, f, sum) : sum;
  }
  sum = wave_sum(sum);
  if (tid % kWave == 0) s_red[1][wave] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += s_red[1][w];

  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (r + x * kRows < runs) acc += early[x] * s_f[r + x * kRows];
#pragma unroll 4
  for (int s = r + 4 * kRows; s < runs; s += kRows) acc += o[int64_t(s) * step] * s_f[s];
  if (r < kRows) s_acc[r][c] = acc;
  __syncthreads();
  if (tid >= kLanes) return;
  acc = s_acc[0][c];
#pragma unroll 8
  for (int x = 1; x < kRows; ++x) acc += s_acc[x][c];
  const float k = sum == 0.f ? 0.f : (p.v_scale ? p.v_scale[row % p.hq / (p.hq / p.hk)] : 1.f) / sum;
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = sum == 0.f ? 0u : pack2<T>(acc[2 * i] * k, acc[2 * i + 1] * k);
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + row * p.d + blockIdx.y * DIMS + c * 4) = w;
  if (p.lse && c == 0 && blockIdx.y == 0) p.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

// How the tokens of the longest sequence are cut into runs, by what was
// measured (us of a call in a graph, bf16, 28 heads of 128 on 4 unless said):
//   - up to 512 tokens one run: a second launch costs more than it saves (200
//     tokens 6.5 against 8.6; but 1024 13.3 against 8.8); up to 1024 where
//     there are 64 blocks without cutting (32 sequences of 1000: 15.7, 20.8);
//   - one sequence: 512 blocks (131072 tokens 55.6; 57.1 with 1024, 60 with 2048);
//   - many: up to 2048 blocks, which even out different lengths (24 sequences
//     of up to 6900, 16 heads of 64 each: 73 against 82 with 1024 and 88 with
//     512; equal ones do not care, 16 of 65536: 369, 379 with 4096);
//   - and at least a tile for each wave of a block, two where blocks abound.
struct Plan {
  int tiles_per_run, runs, waves;
};
Plan plan(int64_t batch, int64_t hq, int64_t hk, int64_t span, bool four) {
  const int64_t tiles = (span + kTile - 1) / kTile;
  const int64_t blocks = batch * hk * ((hq / hk + 15) / 16);
  // 4 bits, up to 128 dims, fewer than 64 blocks: sixteen waves have 24 tiles sooner than two launches (28 heads on 4,
  // 760 tokens: 1 sequence 9.8 us against 10.1, 8 sequences 10.0 against 12.6, with masses 11.6 and 14.0, but 1 sequence with
  // masses 11.4 against 10.6; 1000 tokens 9.9 against 9.3).  From 64 blocks on eight waves are one launch too, and sooner (64
  // sequences 11.0 against 12.3, 200 29.7 against 41.1).
  if (four && blocks < 64 && tiles > 16 && tiles <= 24) return {int(tiles), 1, 16};
  if (tiles <= (blocks >= 64 ? 32 : 16)) return {int(tiles), 1, tiles > 4 ? 8 : 4};
  const int64_t want = (std::min<int64_t>(2048, 512 * batch) + blocks - 1) / blocks;
  int64_t per = std::max<int64_t>(blocks <= 16 ? 4 : 8, (tiles + want - 1) / want);
  per = (per + 3) / 4 * 4;
  return {int(per), int((tiles + per - 1) / per), 4};
}

// Tokens from the first one's tile on that a sequence can span.
int64_t span_of(int64_t max_length, int64_t window) {
  return window > 0 && window < max_length - kTile ? window + kTile : max_length;
}

// Where a call's workspace holds what, in floats.
struct Layout {
  bool whole;                     // one launch writes all; with masses the scores are in its blocks' LDS
  int64_t part_o, scores, end, stride;
};
Layout layout(const Plan& c, int64_t batch, int64_t hq, int64_t hk, int64_t d, bool mass) {
  const int64_t rows = batch * hq;
  Layout l;
  l.stride = int64_t(c.runs) * c.tiles_per_run * kTile;
  const int64_t lds = c.waves * 16 * (d + 4 + 2) + 64 + hq / hk * l.stride;
  l.whole = c.runs == 1 && (!mass || (hq / hk <= 16 && lds * int64_t(sizeof(float)) <= 160 * 1024));
  l.part_o = l.whole ? 0 : (rows * c.runs * 2 + 63) / 64 * 64;
  l.scores = l.whole ? 0 : l.part_o + (mass ? (rows * c.runs * d + 63) / 64 * 64 : rows * c.runs * d);
  l.end = l.scores + (mass && !l.whole ? rows * l.stride : 0);
  return l;
}

template <class T, int DIMS, int THREADS, bool MASS>
void launch_join(const AttendParams& p, const Plan& c, const Layout& l, float* ws, hipStream_t stream) {
  const int64_t rows = int64_t(p.batch) * p.hq, y = p.d / DIMS;
  const int64_t blocks = MASS ? int64_t(p.batch) * p.hk * ((l.stride + 2 * THREADS - 1) / (2 * THREADS)) : 0;
  attend_join_kernel<T, DIMS, THREADS, MASS><<<dim3(unsigned(rows + (blocks + y - 1) / y), unsigned(y)), dim3(THREADS), c.runs * sizeof(float), stream>>>(
      p, c.runs, ws + l.part_o, ws, ws + l.scores, l.stride);
}

template <class T, Held C, int D, int W, bool UNI, bool MASS>
hipError_t launch_form(const AttendParams& p, const Plan& c, hipStream_t stream) {
  const Layout l = layout(c, p.batch, p.hq, p.hk, D, MASS);
  float* ws = static_cast<float*>(p.workspace);
  // Blocks go to the eight XCDs in turn: with an odd count of them a sequence, the
  // runs that short sequences lack are missing from all alike (16 sequences of
  // 1 to 65536 tokens in 32 runs 246 us, with a block more 221).  One sequence
  // lacks none, and its blocks are as many as fill the chip evenly (131072
  // tokens e4m3 31 us, with a block more 36).
  const dim3 grid(unsigned(p.batch > 1 ? c.runs | 1 : c.runs), unsigned(p.hk * ((p.hq / p.hk + 15) / 16)), unsigned(p.batch));
  const size_t lds = MASS && l.whole ? size_t(p.hq / p.hk * l.stride) * sizeof(float) : 0;
  attend_kernel<T, C, D, W, UNI, MASS><<<grid, dim3(64 * W), lds, stream>>>(p, c.tiles_per_run, c.runs, ws + l.part_o, ws, ws + l.scores, l.whole);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || l.whole) return e;
  // Few rows: more blocks, each of a part of the dims (28 rows, 256 runs of 128
  // dims 5.1 -> 2.9 us); many rows need no more blocks (896 rows, 4 runs: 5 us more).
  if (int64_t(p.batch) * p.hq < 256) launch_join<T, 32, 512, MASS>(p, c, l, ws, stream);
  else launch_join<T, D, 256, MASS>(p, c, l, ws, stream);
  return hipGetLastError();
}

template <class T, Held C, int D, bool MASS>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  constexpr bool kFour = C == Held::kE2m1 && D <= 128;
  const Plan c = plan(p.batch, p.hq, p.hk, span_of(p.max_length, p.window), kFour);
  if constexpr (kFour)
    if (c.waves == 16)
      return p.page % kTile == 0 ? launch_form<T, C, D, 16, true, MASS>(p, c, stream) : launch_form<T, C, D, 16, false, MASS>(p, c, stream);
  if (p.page % kTile == 0)
    return c.waves == 8 ? launch_form<T, C, D, 8, true, MASS>(p, c, stream) : launch_form<T, C, D, 4, true, MASS>(p, c, stream);
  return c.waves == 8 ? launch_form<T, C, D, 8, false, MASS>(p, c, stream) : launch_form<T, C, D, 4, false, MASS>(p, c, stream);
}

template <class T, Held C, bool MASS>
hipError_t launch_dim(const AttendParams& p, hipStream_t stream) {
  switch (p.d) {
    case 64: return launch<T, C, 64, MASS>(p, stream);
    case 96: return launch<T, C, 96, MASS>(p, stream);
    case 128: return launch<T, C, 128, MASS>(p, stream);
    case 192: return launch<T, C, 192, MASS>(p, stream);
    case 256: return launch<T, C, 256, MASS>(p, stream);
  }
  return hipErrorInvalidValue;
}

template <Held C, bool MASS>
hipError_t launch_type(const AttendParams& p, hipStream_t stream) {
  return p.type == ServeType::kBf16 ? launch_dim<Bf16, C, MASS>(p, stream) : launch_dim<F16, C, MASS>(p, stream);
}

}  // namespace
}  // namespace cp
