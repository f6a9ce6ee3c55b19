// A few rows times 4-bit weights with group scales:
//   y[i, n] = xs_i sum_g s[n, g] ( sum_{k in g} x[i, k] c[n, k]  -  z[n, g] sum_{k in g} x[i, k] ).
//
// Bound by the weights' bytes.  A code's nibble, alone in a byte, *is* the
// e4m3 value c / 512 (subnormals below 8, the first exponent from 8 on), so
// one conversion instruction widens two codes exactly and the matrix cores
// multiply them; the factor 512 comes back with the scale.  The sums of x of a
// group come from the same instruction with a matrix of ones.  All sums are
// float32.
//
// A lane loads 16 bytes of one output's codes, 32 k: where groups are multiples
// of 128 that is how the products take them (lane group g holds k = 32 g + 8 j
// at step j); smaller groups need each step's 32 k from one group, so the four
// lane groups exchange their words first (k = 32 j + 8 g).
//
// Two kernels.  Few rows or outputs: a wave works on 16 outputs and 16 rows,
// the block's waves take runs of 128 k in turn and their sums meet in LDS.
// More rows: see w4_wide_kernel.
#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// a[d] of lane group r <-> a[r] of lane group d.
__device__ __forceinline__ void transpose4(uint32_t* a) {
  auto s = __builtin_amdgcn_permlane32_swap(a[0], a[2], false, false);
  a[0] = s[0];
  a[2] = s[1];
  s = __builtin_amdgcn_permlane32_swap(a[1], a[3], false, false);
  a[1] = s[0];
  a[3] = s[1];
  s = __builtin_amdgcn_permlane16_swap(a[0], a[1], false, false);
  a[0] = s[0];
  a[1] = s[1];
  s = __builtin_amdgcn_permlane16_swap(a[2], a[3], false, false);
  a[2] = s[0];
  a[3] = s[1];
}

// Eight codes (a word) as the operand's k order 0 2 4 6 1 3 5 7.
template <class T>
__device__ __forceinline__ u32x4 codes(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  return u32x4{widen2<T, false>(lo), widen2<T, true>(lo), widen2<T, false>(hi), widen2<T, true>(hi)};
}

// Eight x from element i on, in the same order.
template <class T>
__device__ __forceinline__ u32x4 order(u32x4 w) {
  return u32x4{__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u),
               __builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
}
// Eight x as they are stored, and as the operand.
template <bool X8>
struct RawX {
  u32x4 w;
  __device__ __forceinline__ void load(const uint8_t* x, unsigned element) {
    if constexpr (X8) {
      const u32x2 v = *reinterpret_cast<const u32x2*>(x + element);
      w[0] = v[0];
      w[1] = v[1];
    } else {
      w = *reinterpret_cast<const u32x4*>(x + 2 * element);
    }
  }
  // What another lane loaded.
  __device__ __forceinline__ void take(int lane) {
#pragma unroll
    for (int e = 0; e < (X8 ? 2 : 4); ++e) w[e] = uint32_t(__builtin_amdgcn_ds_bpermute(4 * lane, int(w[e])));
  }
  // Zero where !inside: the codes that meet it are another k's.
  template <class T>
  __device__ __forceinline__ u32x4 operand(bool inside = true) const {
    u32x4 r;
    if constexpr (X8) {
      const uint32_t even = __builtin_amdgcn_perm(w[1], w[0], 0x06040200u), odd = __builtin_amdgcn_perm(w[1], w[0], 0x07050301u);
      r = u32x4{widen2<T, false>(even), widen2<T, true>(even), widen2<T, false>(odd), widen2<T, true>(odd)};
    } else {
      r = order<T>(w);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = inside ? r[e] : 0u;
    return r;
  }
};

// The loads above stay above: the compiler would move a load that the next
// turn of a loop uses to where it uses it.
__device__ __forceinline__ void keep_loads_here() { asm volatile("" ::: "memory"); }

// A barrier for data in LDS only, so that loads from memory stay under way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// One y (without x's scale) as the formula says, code by code.  The kernels take
// the zero points off the groups' sums, which is another thing where x is
// infinite, or a sum past float32's range; such results are found again here.
// NaN ends it with its group.  (64 x 3584 x 28672: 33 us, a row with an infinity
// 0.12 ms, 64 of them 2.1, 64 rows of NaN 0.11.)
template <class T>
__device__ __forceinline__ float by_formula(const W4Params& p, int64_t m, int64_t n) {
  const int groups = p.k / p.group;
  const uint16_t* x = static_cast<const uint16_t*>(p.x) + m * p.k;
  const uint8_t* w = p.weight + n * (p.k / 2);
  float y = 0.f;
  for (int i = 0; i < groups && y == y; ++i) {
    const float zero = p.zero ? float(p.zero[n * groups + i]) : 8.f;
    float sum = 0.f;
    // (One load of x at a time: the kernels' registers are for their own loop.)
#pragma unroll 1
    for (int j = i * p.group; j < (i + 1) * p.group; j += 8) {
      const uint32_t eight = *reinterpret_cast<const uint32_t*>(w + j / 2);
      float v[8];
      load8<T>(x, j, v);
#pragma unroll
      for (int l = 0; l < 8; ++l) sum = fmaf(v[l], float(eight >> 4 * l & 15) - zero, sum);
    }
    y = fmaf(sum, load1<T>(p.scale, n * groups + i), y);
  }
  return y;
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }

// SPAN: steps of 32 k between two groups' ends, 4, 2 or 1 (group a multiple of
// 128, of 64, of 32).
//
// A lane's loads are never conditional: past the end of x, of the rows or of k
// they read the last ones again, so that the next run's are under way while
// this one's are used.  Results of rows and outputs that do not exist are not
// stored, and x is zero past k.  Addresses are a wave's base plus 32 bits of a
// lane's own; what is loaded stays as it is stored until it is used.

// r-th run of 32 k -> its group.
__device__ __forceinline__ int group_of(const W4Params& p, int r) {
  return int(unsigned((uint64_t(r) * p.group_magic) >> 32) + unsigned(r) * p.group_one);
}

__device__ __forceinline__ uint32_t from_lane(uint32_t v, int lane) {
  return uint32_t(__builtin_amdgcn_ds_bpermute(4 * lane, int(v)));
}

// The scales and zero points of a lane's output.  A lane's load of two bytes
// and one touches as many cache lines as one of its codes, so lane group g
// loads those of the g-th of the next four groups that the wave meets (of SPAN
// runs), and they trade.
struct Scales {
  uint16_t s;
  uint8_t z;

  // lane: the output's first group, from the block's first output's on.
  __device__ __forceinline__ void load(const W4Params& p, int64_t n0, unsigned lane, int groups, int run) {
    const int64_t base = n0 * groups;
    const unsigned at = lane + unsigned(min(group_of(p, run), groups - 1));
    s = (static_cast<const uint16_t*>(p.scale) + base)[at];
    // Without zero points a byte of the scales is read in their place and dropped.
    z = ((p.zero ? p.zero : static_cast<const uint8_t*>(p.scale)) + base)[at];
  }
  // The d-th group's of output c, which lane 4 c + d has, -> all[d].
  __device__ __forceinline__ void trade(const W4Params& p, int c, uint32_t* all) const {
    const uint32_t v = s | uint32_t(p.zero ? z : 8) << 16;
#pragma unroll
    for (int d = 0; d < 4; ++d) all[d] = from_lane(v, 4 * c + d);
  }
};

// The 32 codes of lane group g at a run of 128 k; lane: the output's first byte.
__device__ __forceinline__ u32x4 load_codes(const W4Params& p, int64_t n0, unsigned lane, int kb, int g) {
  const int last = (p.k - 1) / 128 * 128, at = min(kb, last);
  const uint8_t* base = p.weight + n0 * (p.k / 2) + at / 2;
  return *reinterpret_cast<const u32x4*>(base + (lane + unsigned(min(g * 32, p.k - 32 - at)) / 2));
}

template <class T, bool TRADE>
__device__ __forceinline__ void operands(u32x4 w, u32x4* a) {
  uint32_t v[4] = {w[0], w[1], w[2], w[3]};
  if constexpr (TRADE) transpose4(v);
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = codes<T>(v[j]);
}

// Neighbouring lanes' x -> x[0 .. SHARE - 1] of them all.
template <int SHARE>
__device__ __forceinline__ void spread(u32x4 v, u32x4* x) {
  auto moved = [](uint32_t w, auto ctrl) { return uint32_t(__builtin_amdgcn_mov_dpp(int(w), decltype(ctrl)::value, 0xf, 0xf, false)); };
  if constexpr (SHARE == 1) x[0] = v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (SHARE == 2) {
      x[0][e] = moved(v[e], std::integral_constant<int, 0xa0>());   // quad: 0 0 2 2
      x[1][e] = moved(v[e], std::integral_constant<int, 0xf5>());   // quad: 1 1 3 3
    }
    if constexpr (SHARE == 4) {
      x[0][e] = moved(v[e], std::integral_constant<int, 0x00>());   // quad: 0 0 0 0
      x[1][e] = moved(v[e], std::integral_constant<int, 0x55>());   // quad: 1 1 1 1
      x[2][e] = moved(v[e], std::integral_constant<int, 0xaa>());   // quad: 2 2 2 2
      x[3][e] = moved(v[e], std::integral_constant<int, 0xff>());   // quad: 3 3 3 3
    }
  }
}

// Up to 16 rows.  A wave works on 16 RT outputs, whose x it reads from the
// caches and puts in order once for all of them, at every waves-th run of 128
// k; the sums of the block's waves meet in LDS.
//
// What a compute unit can fill bounds it, and at 64 bytes a cycle a run's x,
// 16 rows of it, takes 64 cycles beside some 95 of 16 outputs' codes.  Up to 16
// / SHARE rows, SHARE neighbouring lanes hold one row: each loads its share of
// the row's x once and they pass it on; row r of x is then the product's rows
// SHARE r to SHARE r + SHARE - 1, all alike.  At 1 x 3584 x 28672, groups of
// 128, 14.5 us (3.6 TB/s) over weights that pass the caches, 12.1 where they
// stay; at 16 rows 17.9 (3.0 TB/s) and 15.9.
template <class T, bool X8, int SPAN, int RT, int SHARE>
__global__ __launch_bounds__(SHARE == 4 ? 1024 : 512) void w4_few_kernel(W4Params p, int64_t first_block) {
  constexpr int kGroups = 4 / SPAN;
  constexpr bool kDirect = SPAN == 4 && SHARE == 4;
  extern __shared__ float s_part[];               // [waves][RT][16][17]
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
  const int c = lane % 16, g = lane / 16;
  const int64_t n0 = (first_block + blockIdx.x) * (16 * RT), m0 = int64_t(blockIdx.y) * 16;
  const int groups = p.k / p.group;
  const uint32_t one = pack2<T>(1.f, 1.f);
  const u32x4 ones = {one, one, one, one};
  unsigned row[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) row[i] = unsigned(min(int64_t(i * 16 + lane / 4), p.n - 1 - n0));
  const int own = 4 * c + g;                      // the lane that loads what this one needs
  const unsigned xrow = unsigned(min(int64_t(kDirect ? c / SHARE : lane / (4 * SHARE)), p.m - 1 - m0)) * unsigned(p.k);
  const uint8_t* xbase = static_cast<const uint8_t*>(p.x) + m0 * p.k * (X8 ? 1 : 2);
  f32x4 y[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) y[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Step j's k of this lane; the first of its j-th load of x.
  auto k_of = [&](int kb, int j) { return kb + (kDirect ? g * 32 + j * 8 : j * 32 + g * 8); };
  auto k_load = [&](int kb, int j) { return kDirect ? k_of(kb, c % SHARE) : kb + j * SHARE * 32 + lane % (4 * SHARE) * 8; };
  struct Stage {
    u32x4 w[RT];
    RawX<X8> x[4 / SHARE];
  } stage;
  Scales scales[RT];
  const int step = waves * 128;
  // What a run needs, on its way while the run before is worked on.
  auto load = [&](Stage& s, int kb) {
#pragma unroll
    for (int i = 0; i < RT; ++i) s.w[i] = load_codes(p, n0, row[i] * unsigned(p.k / 2), kb, lane % 4);
#pragma unroll
    for (int j = 0; j < 4 / SHARE; ++j) s.x[j].load(xbase, xrow + unsigned(min(k_load(kb, j), p.k - 8)));
    keep_loads_here();
  };
  auto load_scales = [&](int kb) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
      scales[i].load(p, n0, row[i] * unsigned(groups), groups, (kb + lane % 4 / kGroups * step) / 32 + lane % kGroups * SPAN);
    keep_loads_here();
  };
  // Run t of SPAN at kb; all: their scales and zero points.
  auto use = [&](Stage& s, int kb, int t, uint32_t (*all)[4], bool more, bool more_scales) {
    u32x4 a[RT][4], b[4];
    float sc[RT][kGroups], z[RT][kGroups];
#pragma unroll
    for (int j = 0; j < 4 / SHARE; ++j) {
      if (!kDirect) s.x[j].take(own);
      spread<SHARE>(s.x[j].template operand<T>(SPAN == 4 || k_of(kb, j * SHARE + c % SHARE) < p.k), b + j * SHARE);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s.w[i][e] = from_lane(s.w[i][e], own);
      operands<T, !kDirect>(s.w[i], a[i]);
#pragma unroll
      for (int h = 0; h < kGroups; ++h) {
        const uint32_t v = all[i][t * kGroups + h];
        const float scale = unpack2<T>(v).x;
        sc[i][h] = 512.f * scale;
        z[i][h] = -scale * float(v >> 16);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more_scales) load_scales(kb + SPAN * step);
    if (more) load(s, kb + step);
#pragma unroll
    for (int h = 0; h < kGroups; ++h) {
      f32x4 sum = {0.f, 0.f, 0.f, 0.f}, acc[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = h * SPAN; j < (h + 1) * SPAN; ++j) {
        sum = mfma32<T>(b[j], ones, sum);
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[i] = mfma32<T>(b[j], a[i][j], acc[i]);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int r = 0; r < 4; r += SHARE) y[i][r] = fmaf(sc[i][h], acc[i][r], fmaf(z[i][h], sum[r], y[i][r]));
    }
  };
  int kb = wave * 128;
  load_scales(kb);
  load(stage, kb);
  while (kb < p.k) {
    uint32_t all[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i) scales[i].trade(p, c, all[i]);
#pragma unroll
    for (int t = 0; t < SPAN; ++t, kb += step) {
      if (kb >= p.k) break;
      use(stage, kb, t, all, kb + step < p.k, t == 0 && kb + SPAN * step < p.k);
    }
  }

  // y[i][r] of lane (g, c): output 16 i + c of row 4 g + r.
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int r = 0; r < 4; r += SHARE) s_part[((wave * RT + i) * 16 + g * 4 + r) * 17 + c] = y[i][r];
  __syncthreads();
  for (int e = threadIdx.x; e < RT * 256 / SHARE; e += blockDim.x) {
    const int i = e / 16 % RT, mr = e / (16 * RT) * SHARE;
    const int64_t m = m0 + mr / SHARE, n = n0 + i * 16 + e % 16;
    if (m >= p.m || n >= p.n) continue;
    float v = 0.f;
    for (int x = 0; x < waves; ++x) v += s_part[((x * RT + i) * 16 + mr) * 17 + e % 16];
    if (X8) v *= p.x_scale[m];
    else if (!is_finite(v)) v = by_formula<T>(p, m, n);
    if (p.y_type == ServeType::kF32) store1<F32>(p.y, m * p.n + n, v);
    else store1<T>(p.y, m * p.n + n, v);
  }
}

// Scales and zero points go to LDS some groups at a time: a lane needs those
// of one output, so its own loads would touch a cache line each, as many as
// its codes do.  Row o of `rows` outputs from n0 on, groups g0 .. g0 + count - 1.
template <int PITCH>
__device__ __forceinline__ void keep_scales(const W4Params& p, int64_t n0, int rows, int g0, int count, uint16_t* s, uint8_t* z) {
  const int groups = p.k / p.group, last = int(min(int64_t(rows), p.n - n0)) - 1;
  for (int i = threadIdx.x % kWave; i < count; i += kWave) {
#pragma unroll 4
    for (int o = threadIdx.x / kWave; o < rows; o += blockDim.x / kWave) {
      const int64_t at = (n0 + min(o, last)) * groups + g0 + i;
      s[o * PITCH + i] = static_cast<const uint16_t*>(p.scale)[at];
      z[o * PITCH + i] = p.zero ? p.zero[at] : uint8_t(8);
    }
  }
}
template <class T>
__device__ __forceinline__ float widen1(uint16_t bits) { return unpack2<T>(bits).x; }

// Sum over the 4, 8 or 16 neighbouring lanes that hold 32 SPAN k; they all get it.
template <int SPAN>
__device__ __forceinline__ float span_sum(float x) {
  auto moved = [](float v, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
  x += moved(x, std::integral_constant<int, 0xb1>());                      // quad: 1 0 3 2
  x += moved(x, std::integral_constant<int, 0x4e>());                      // quad: 2 3 0 1
  if constexpr (SPAN >= 2) x += moved(x, std::integral_constant<int, 0x141>());   // half rows reversed
  if constexpr (SPAN >= 4) x += moved(x, std::integral_constant<int, 0x140>());   // rows reversed
  return x;
}

// c + the two products of a packed pair of T with 1.
template <class T>
__device__ __forceinline__ float add2(uint32_t w, float c);
template <>
__device__ __forceinline__ float add2<Bf16>(uint32_t w, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{(__bf16)1.f, (__bf16)1.f}, c, false);
}
template <>
__device__ __forceinline__ float add2<F16>(uint32_t w, float c) {
  return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), f16x2{(_Float16)1.f, (_Float16)1.f}, c, false);
}

// 16 MT rows of x by 128 outputs.  x would be read once per 16 outputs from the
// caches if each wave did so by itself, many times the weights' bytes; here
// the block brings 256 k of it to LDS at a time, as operands, with the groups'
// sums beside them, while it works on the 256 before.  Waves: 8 by outputs (16
// each) times 2 by k; codes are loaded two turns ahead.
//
// At 64 x 3584 x 28672, groups of 64, 32 us (1.9 TB/s of codes, 410 TFLOP/s).
// Nothing is full: of a SIMD's cycles 55 % issue vector instructions (153 a wave
// and turn, 28 of them to widen the codes, beside 20 matrix ones), the matrix
// cores work in 30 %, LDS in 32 %; the waves wait in 44 % of theirs, at the turn's
// barrier among others, with no second block on the compute unit.  32 outputs a
// wave read LDS half as often but do not fit the registers of 16 waves (44 us; 40
// with 8 waves), turns of 512 k change nothing (34).
constexpr int kWideRows = 128;
constexpr int kWideGroups = 64;                   // whose scales are in LDS at a time
template <class T, bool X8, int SPAN, int MT>
__global__ __launch_bounds__(1024) void w4_wide_kernel(W4Params p, int64_t first_block) {
  constexpr int kGroups = 4 / SPAN, kPitch = kWideGroups + 2, kMine = MT / 2;
  __shared__ u32x4 s_x[2][2][4][MT][kWave];       // [turn % 2][half][step][row tile][lane]
  __shared__ uint16_t s_scale[kWideRows * kPitch];
  __shared__ uint8_t s_zero[kWideRows * kPitch];
  __shared__ float s_sum[2][2][MT][kWave];        // [turn % 2][half][row tile][group, row]
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c = lane % 16, g = lane / 16, half = wave / 8;
  const int64_t first = (first_block + blockIdx.x) * kWideRows, out0 = first + wave % 8 * 16, n0 = min(out0, p.n - 1);
  const int64_t m0 = int64_t(blockIdx.y) * (16 * MT);
  const int turns = (p.k + 255) / 256, last_group = p.k / p.group - 1;
  const unsigned row = unsigned(min(int64_t(c), p.n - 1 - n0)) * unsigned(p.k / 2);
  f32x4 y[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) y[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // This thread's share of a turn's x: 8 k from 8 q on of a half, row xr of
  // every other tile.  A wave holds four rows' 128 k, whose operands would
  // fall into the same banks; so the rows of a step's lane group change places.
  const int q = tid % 16, xhalf = wave / 4 % 2, xr = tid / 16 % 16, xt = wave / 8, xk = xhalf * 128 + q * 8;
  const int xj = SPAN < 4 ? q / 4 : q % 4, xg = SPAN < 4 ? q % 4 : q / 4;
  const int slot = xg * 16 + (xr ^ (xj * 4 + xg));
  const uint8_t* xbase = static_cast<const uint8_t*>(p.x) + m0 * p.k * (X8 ? 1 : 2);
  unsigned xrow[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) xrow[i] = unsigned(min(int64_t((2 * i + xt) * 16 + xr), p.m - 1 - m0)) * unsigned(p.k);
  // Groups past a run's last are multiplied by zero.
  for (int i = tid; i < 2 * 2 * MT * kWave; i += 1024) (&s_sum[0][0][0][0])[i] = 0.f;
  __syncthreads();
  RawX<X8> xv[2][kMine];
  u32x4 w[2];
  auto load_x = [&](RawX<X8>* v, int turn) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) v[i].load(xbase, xrow[i] + unsigned(min(turn * 256 + xk, p.k - 8)));
    keep_loads_here();
  };
  auto load_w = [&](u32x4* v, int turn) {
    *v = load_codes(p, n0, row, turn * 256 + half * 128, g);
    keep_loads_here();
  };
  auto keep_x = [&](auto whole, const RawX<X8>* raw, int buf, int turn) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      u32x4 v = raw[i].template operand<T>(whole || turn * 256 + xk < p.k);
      s_x[buf][xhalf][xj][2 * i + xt][slot] = v;
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) s = add2<T>(v[e], s);
      s = span_sum<SPAN>(s);
      if (q % (4 * SPAN) == 0) s_sum[buf][xhalf][2 * i + xt][q / (4 * SPAN) * 16 + xr] = s;
    }
  };
  int g0 = 0;                                     // first group whose scales are in LDS
  // One turn: its x is in s_x[buf], its codes in w[buf]; the turn after's x is
  // in xv[1 - buf] or on its way.
  auto turn_of = [&](auto more, int buf, int turn) {
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = w[buf][j];
    if constexpr (SPAN < 4) transpose4(v);
    auto place = [&](int h) {
      return (wave % 8 * 16 + c) * kPitch + min(group_of(p, turn * 8 + half * 4 + h * SPAN), last_group) - g0;
    };
    float scale[kGroups];
#pragma unroll
    for (int h = 0; h < kGroups; ++h) scale[h] = 512.f * widen1<T>(s_scale[place(h)]);
    // Lane group g gives the zero points of the run's group g.
    const int own = place(min(g, kGroups - 1));
    const float zero = g < kGroups ? -widen1<T>(s_scale[own]) * float(s_zero[own]) : 0.f;
    __builtin_amdgcn_sched_barrier(0);
    if (more || turn + 2 < turns) {
      // x first: what waits for it, at the end of the next turn, then does not
      // wait for the codes of the turn after.
      load_x(xv[buf], turn + 2);
      load_w(&w[buf], turn + 2);
    }
#pragma unroll
    for (int h = 0; h < kGroups; ++h) {
      f32x4 acc[MT];
#pragma unroll
      for (int j = h * SPAN; j < (h + 1) * SPAN; ++j) {
        const u32x4 a = codes<T>(v[j]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[t] = mfma32<T>(s_x[buf][half][j][t][g * 16 + (c ^ (j * 4 + g))], a, j == h * SPAN ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[t]);
      }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) y[t][r] = fmaf(scale[h], acc[t][r], y[t][r]);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) y[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(s_sum[buf][half][t][g * 16 + c], zero, y[t], 0, 0, 0);
    if (more || turn + 1 < turns) keep_x(more, xv[1 - buf], 1 - buf, turn + 1);
    lds_barrier();
  };
  load_x(xv[0], 0);
  load_w(&w[0], 0);
  load_x(xv[1], 1);
  load_w(&w[1], 1);
  keep_x(std::false_type(), xv[0], 0, 0);
  lds_barrier();
  // kWideGroups groups are `block` turns, an even number (group / 4).
  const int block = kWideGroups * p.group / 256;
  int turn = 0, stop = 0;
  auto next_scales = [&] {
    stop = turn + block;
    g0 = group_of(p, turn * 8);
    keep_scales<kPitch>(p, first, kWideRows, g0, min(kWideGroups, last_group + 1 - g0), s_scale, s_zero);
    lds_barrier();
  };
  // While two more turns are certain nothing about the loads is conditional, so
  // that each wait is for just what it needs.
  while (turn + 4 <= turns) {
    next_scales();
    const int end = min(stop, (turns - 2) / 2 * 2);
    for (; turn < end; turn += 2) {
      turn_of(std::true_type(), 0, turn);
      turn_of(std::true_type(), 1, turn + 1);
    }
  }
  for (; turn < turns; turn += 2) {
    if (turn == stop) next_scales();
    turn_of(std::false_type(), 0, turn);
    if (turn + 1 < turns) turn_of(std::false_type(), 1, turn + 1);
  }

  // The halves meet.  y[t][r] of lane (g, c): output c of row 16 t + 4 g + r.
  f32x4* part = &reinterpret_cast<f32x4*>(&s_x[0][0][0][0][0])[wave % 8 * (MT * kWave) + lane];
  if (half == 1)
#pragma unroll
    for (int t = 0; t < MT; ++t) part[t * kWave] = y[t];
  __syncthreads();
  if (half == 1) return;
  const int64_t n = out0 + c;
  auto store = [&](int64_t m, float v) {
    if (p.y_type == ServeType::kF32) store1<F32>(p.y, m * p.n + n, v);
    else store1<T>(p.y, m * p.n + n, v);
  };
  unsigned again = 0;                             // bit 4 t + r
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const f32x4 o = part[t * kWave];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t m = m0 + t * 16 + g * 4 + r;
      if (m >= p.m || n >= p.n) continue;
      float v = y[t][r] + o[r];
      if (X8) v *= p.x_scale[m];
      else again |= unsigned(!is_finite(v)) << (4 * t + r);
      store(m, v);
    }
  }
  for (; !X8 && again; again &= again - 1) {
    const int i = __builtin_ctz(again);
    const int64_t m = m0 + i / 4 * 16 + g * 4 + i % 4;
    store(m, by_formula<T>(p, m, n));
  }
}

template <class T, bool X8, int SPAN, int MT>
hipError_t launch_wide(const W4Params& p, hipStream_t stream) {
  const unsigned row_blocks = unsigned((p.m + 16 * MT - 1) / (16 * MT));
  return launch_blocks((p.n + kWideRows - 1) / kWideRows, 1024, [&](int64_t first, unsigned blocks) {
    w4_wide_kernel<T, X8, SPAN, MT><<<dim3(blocks, row_blocks), dim3(1024), 0, stream>>>(p, first);
  });
}

template <class T, bool X8, int SPAN, int RT, int SHARE>
hipError_t launch_few(const W4Params& p, hipStream_t stream) {
  const int most = RT == 4 ? 4 : SHARE == 4 && p.k >= 8192 ? 16 : 8, waves = std::min(most, (p.k + 127) / 128);
  const unsigned row_blocks = unsigned((p.m + 15) / 16);
  return launch_blocks((p.n + 16 * RT - 1) / (16 * RT), kWave * waves, [&](int64_t first, unsigned blocks) {
    w4_few_kernel<T, X8, SPAN, RT, SHARE><<<dim3(blocks, row_blocks), dim3(kWave * waves), size_t(waves) * RT * 272 * sizeof(float),
                                            stream>>>(p, first);
  });
}

// Which kernel (rows x k x outputs, groups of 128, bf16, over weights that
// together pass the caches; us of one call in a graph, both sides of each rule
// from one sweep; a tile is 16 rows by 16 outputs):
//   - more than 16 rows and many outputs: the wide one, whose time hardly
//     depends on either up to a block a compute unit, while that of the other
//     grows with rows x outputs.  With 32 rows a block they meet near 655360
//     (32x3584x28672 23.5 against 28.7, 64x3584x12288 21.2 against 22.6,
//     64x1792x16384 13.8 against 18.0; but 32x3584x18000 21.4 against 20.5,
//     48x3584x12288 21.0 against 19.7), while its blocks are not more than
//     compute units; with 64 near 2^20 (64x3584x28672 31.3 against 46.2; but
//     48x3584x18000 29.9 against 26.7);
//   - up to 4 rows, lanes share x four ways (1x3584x4608 5.6 against 6.3 two ways
//     and 7.1 with none, 1x14336x3584 9.1, 13.9 and 15.1, 1x3584x28672 14.4, 16.0
//     and 21.5); up to 8 rows, two ways (8x3584x28672 16.3 against 17.5 with none,
//     8x2048x12000 6.8 and 7.5);
//   - 16 outputs a wave while there are fewer tiles than compute units
//     (16x14336x3584 15.5, with 32 19.5); then 32 (16x3584x4608 7.1, with 16 8.4,
//     with 64 11.4; 24x3584x4608 8.8, with 64 11.3; 48x14336x3584 27.0, with 64
//     32.1); and 64 from 1536 tiles on (16x3584x28672 17.9, with 32 19.5;
//     64x2048x12000 15.8 and 16.0).  That bound is right for 16 rows only: with 17
//     to 48 rows 32 outputs would be the faster up to some 3000 tiles
//     (48x3584x12288 19.7, with 64 21.7, groups of 64 22.4 and 24.6, of 32 25.1 and
//     27.6; 32x3584x18000 20.5 and 22.7; 48x2048x12000 13.7 and 15.1);
//   - 8 waves a block, 16 for a long k (1x14336x3584 9.2 against 12.7 with 8; but
//     1x3584x28672 19.9 against 14.4), 4 where each holds 64 outputs.
template <class T, bool X8, int SPAN>
hipError_t launch_span(const W4Params& p, hipStream_t stream) {
  const int64_t work = (p.m + 15) / 16 * 16 * p.n;
  if (p.m > 16 && work >= 655360) {
    if (p.m <= 32 || (p.m + 31) / 32 * ((p.n + kWideRows - 1) / kWideRows) <= 256) return launch_wide<T, X8, SPAN, 2>(p, stream);
    if (work >= 1 << 20) return launch_wide<T, X8, SPAN, 4>(p, stream);
  }
  const int64_t tiles = (p.m + 15) / 16 * ((p.n + 15) / 16);
  if (p.m <= 4) return launch_few<T, X8, SPAN, 1, 4>(p, stream);
  if (p.m <= 8) return tiles < 256 ? launch_few<T, X8, SPAN, 1, 2>(p, stream) : launch_few<T, X8, SPAN, 2, 2>(p, stream);
  if (tiles < 256) return launch_few<T, X8, SPAN, 1, 1>(p, stream);
  return tiles <= 1536 ? launch_few<T, X8, SPAN, 2, 1>(p, stream) : launch_few<T, X8, SPAN, 4, 1>(p, stream);
}

template <class T, bool X8>
hipError_t launch_type(const W4Params& p, hipStream_t stream) {
  if (p.group % 128 == 0) return launch_span<T, X8, 4>(p, stream);
  if (p.group % 64 == 0) return launch_span<T, X8, 2>(p, stream);
  return launch_span<T, X8, 1>(p, stream);
}

}  // namespace

hipError_t launch_w4_matvec(const W4Params& p, hipStream_t stream) {
  if (p.type == ServeType::kBf16) return p.x_scale ? launch_type<Bf16, true>(p, stream) : launch_type<Bf16, false>(p, stream);
  return p.x_scale ? launch_type<F16, true>(p, stream) : launch_type<F16, false>(p, stream);
}

}  // namespace cp
