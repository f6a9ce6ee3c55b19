// Attention of one new token of each sequence over a paged key-value cache,
// split over the cache's length and joined:
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),
// j over the sequence's tokens (the last `window` of them), m a running
// maximum; o = 0 and lse = -inf where there is none.
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
// The running maximum moves only when a score passes it by more than 2^8, so
// that the usual tile needs no exchange between lanes and no rescaling.
// p is handed over as two values of the cache's type (its rounding and the
// rest), so no accuracy is lost to it; sums and statistics are float32.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

constexpr int kWaves = 4;
constexpr int kTile = 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// How far a score may pass the running maximum, in powers of two.
constexpr float kSlack = 8.f;

// 32 x 16 pieces of a head's dims held by a lane of the value operand: runs of
// 8, 4 and 2 dims, from 128, 64 and 32 dims of the head.
template <int D>
struct Dims {
  static constexpr int n8 = D / 128, n4 = D % 128 / 64, n2 = D % 64 / 32;
  static constexpr int pairs = D / 32;          // packed pairs a lane holds of a token
  // First dim of pair q of lane c.
  static __device__ __forceinline__ int dim(int q, int c) {
    if (q < 4 * n8) return q / 4 * 128 + c * 8 + q % 4 * 2;
    if (q < 4 * n8 + 2 * n4) return n8 * 128 + c * 4 + (q - 4 * n8) * 2;
    return n8 * 128 + n4 * 64 + c * 2;
  }
};

// A lane's dims of one token's value row, as packed pairs of T.
template <class T, bool C8, int D>
__device__ __forceinline__ void load_value(const uint8_t* row, int c, uint32_t* out) {
  using L = Dims<D>;
  if constexpr (!C8) {
#pragma unroll
    for (int i = 0; i < L::n8; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(row + i * 256 + c * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[4 * i + j] = w[j];
    }
    if constexpr (L::n4) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(row + L::n8 * 256 + c * 8);
      out[4 * L::n8] = w[0];
      out[4 * L::n8 + 1] = w[1];
    }
    if constexpr (L::n2) out[4 * L::n8 + 2 * L::n4] = *reinterpret_cast<const uint32_t*>(row + L::n8 * 256 + L::n4 * 128 + c * 4);
  } else {
#pragma unroll
    for (int i = 0; i < L::n8; ++i) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(row + i * 128 + c * 8);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        out[4 * i + 2 * j] = widen2<T, false>(w[j]);
        out[4 * i + 2 * j + 1] = widen2<T, true>(w[j]);
      }
    }
    if constexpr (L::n4) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(row + L::n8 * 128 + c * 4);
      out[4 * L::n8] = widen2<T, false>(w);
      out[4 * L::n8 + 1] = widen2<T, true>(w);
    }
    if constexpr (L::n2)
      out[4 * L::n8 + 2 * L::n4] = widen2<T, false>(*reinterpret_cast<const uint16_t*>(row + L::n8 * 128 + L::n4 * 64 + c * 2));
  }
}

// Eight dims from dim d on of one token's key row.
template <class T, bool C8>
__device__ __forceinline__ u32x4 load_key(const uint8_t* row, int d) {
  if constexpr (!C8) return *reinterpret_cast<const u32x4*>(row + 2 * d);
  const u32x2 w = *reinterpret_cast<const u32x2*>(row + d);
  return u32x4{widen2<T, false>(w[0]), widen2<T, true>(w[0]), widen2<T, false>(w[1]), widen2<T, true>(w[1])};
}

// One (sequence, key-value head, up to 16 of its query heads, run of tiles).
// Partial results of run s: o [head][D], then m and l, unnormalised.
template <class T, bool C8, int D>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(AttendParams p, int tiles_per_run, int runs, float* part_o,
                                                             float* part_ml) {
  constexpr int kSteps = D / 32;
  using L = Dims<D>;
  __shared__ float s_o[kWaves][16][D + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane % 16, g = lane / 16;
  const int group = p.hq / p.hk, head_tiles = (group + 15) / 16;
  const int run = blockIdx.x, kh = blockIdx.y / head_tiles, h0 = kh * group + blockIdx.y % head_tiles * 16;
  const int heads = min(16, (kh + 1) * group - h0);
  const int b = blockIdx.z;

  int hi = p.lengths[b];
  hi = max(0, int(min(int64_t(hi), p.max_length)));
  const int lo = p.window > 0 ? max(0, hi - p.window) : 0;
  const int tile0 = lo / kTile + run * tiles_per_run;
  const int tile1 = min((hi + kTile - 1) / kTile, tile0 + tiles_per_run);
  const int32_t* table = p.table + int64_t(b) * p.width;
  constexpr int kRow = D * (C8 ? 1 : 2);
  const uint8_t* kc = static_cast<const uint8_t*>(p.k_cache);
  const uint8_t* vc = static_cast<const uint8_t*>(p.v_cache);

  u32x4 q[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    q[j] = u32x4{0, 0, 0, 0};
    if (c < heads)
      q[j] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.q) + (int64_t(b) * p.hq + h0 + c) * D + j * 32 + g * 8);
  }
  const float to_log2 = p.scale * kLog2e * (p.k_scale ? p.k_scale[kh] : 1.f);

  float m = -INFINITY, l = 0.f;
  f32x4 o[2 * L::pairs];
#pragma unroll
  for (int i = 0; i < 2 * L::pairs; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int tile = tile0 + wave; tile < tile1; tile += kWaves) {
    const int t0 = tile * kTile;
    // Lane l finds token l % 32's row; tokens outside [lo, hi) take the
    // nearest one inside (their p is 0, and theirs of V too).
    const int t = min(max(t0 + lane % 32, lo), hi - 1);
    const int pg = t / p.page;
    const unsigned page = min(unsigned(table[pg]), unsigned(p.pages - 1));
    const unsigned my_row = (page * unsigned(p.hk) + unsigned(kh)) * unsigned(p.page) + unsigned(t - pg * p.page);

    u32x4 key[2][kSteps];
    uint32_t val[8][L::pairs];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* r = kc + uint64_t(unsigned(__shfl(int(my_row), i * 16 + c))) * kRow;
#pragma unroll
      for (int j = 0; j < kSteps; ++j) key[i][j] = load_key<T, C8>(r, j * 32 + g * 8);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint8_t* r = vc + uint64_t(unsigned(__shfl(int(my_row), i / 4 * 16 + g * 4 + i % 4))) * kRow;
      load_value<T, C8, D>(r, c, val[i]);
    }

    f32x4 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kSteps; ++j) s[i] = mfma32<T>(key[i][j], q[j], s[i]);
    }
    const bool partial = t0 < lo || t0 + kTile > hi;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[i / 4][i % 4] * to_log2;
    if (partial) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = t0 + i / 4 * 16 + g * 4 + i % 4;
        if (at < lo || at >= hi) {
          x[i] = -INFINITY;
#pragma unroll
          for (int j = 0; j < L::pairs; ++j) val[i][j] = 0;
        }
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m2 = fmaxf(m, top);
      const float f = m2 == m ? 1.f : exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int i = 0; i < 2 * L::pairs; ++i) o[i] *= f;
    }
    u32x4 ph, pl;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float a = exp2f(x[i] - m), e = exp2f(x[i + 1] - m);
      l += a + e;
      ph[i / 2] = pack2<T>(a, e);
      const float2 r = unpack2<T>(ph[i / 2]);
      pl[i / 2] = pack2<T>(a - r.x, e - r.y);
    }
#pragma unroll
    for (int i = 0; i < L::pairs; ++i) {
      u32x4 even, odd;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        even[j] = __builtin_amdgcn_perm(val[2 * j + 1][i], val[2 * j][i], 0x05040100u);
        odd[j] = __builtin_amdgcn_perm(val[2 * j + 1][i], val[2 * j][i], 0x07060302u);
      }
      o[2 * i] = mfma32<T>(even, ph, o[2 * i]);
      o[2 * i] = mfma32<T>(even, pl, o[2 * i]);
      o[2 * i + 1] = mfma32<T>(odd, ph, o[2 * i + 1]);
      o[2 * i + 1] = mfma32<T>(odd, pl, o[2 * i + 1]);
    }
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
  for (int i = 0; i < L::pairs; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int d = L::dim(i, g * 4 + r);
      s_o[wave][c][d] = o[2 * i][r];
      s_o[wave][c][d + 1] = o[2 * i + 1][r];
    }
  __syncthreads();
  const float vs = p.v_scale ? p.v_scale[kh] : 1.f;
  for (int i = threadIdx.x; i < heads * D; i += 64 * kWaves) {
    const int h = i / D, d = i % D;
    float M = s_m[0][h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][h]);
    float acc = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (s_l[w][h] == 0.f) continue;         // a wave without tokens
      const float f = exp2f(s_m[w][h] - M);
      acc = fmaf(s_o[w][h][d], f, acc);
      sum = fmaf(s_l[w][h], f, sum);
    }
    const int64_t row = int64_t(b) * p.hq + h0 + h;
    if (runs == 1) {
      store1<T>(p.out, row * D + d, sum == 0.f ? 0.f : acc / sum * vs);
      if (p.lse && d == 0) p.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
    } else {
      part_o[(row * runs + run) * D + d] = acc;
      if (d == 0) {
        part_ml[(row * runs + run) * 2] = M;
        part_ml[(row * runs + run) * 2 + 1] = sum;
      }
    }
  }
}

// The runs of one (sequence, query head) joined.  The runs' weights are found
// once, in LDS; then D / 4 threads read a run's row and the block's other
// threads read other runs', so a long sequence's rows are in flight together.
constexpr int kJoinThreads = 512;
template <class T, int D>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendParams p, int runs, const float* part_o,
                                                                   const float* part_ml) {
  constexpr int kLanes = D / 4, kRows = kJoinThreads / kLanes;
  extern __shared__ float s_f[];                // [runs] weights
  __shared__ float s_red[kJoinThreads / kWave];
  __shared__ f32x4 s_acc[kRows][kLanes];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  const float2* ml = reinterpret_cast<const float2*>(part_ml) + row * runs;
  float M = -INFINITY;
  for (int s = tid; s < runs; s += kJoinThreads) {
    const float2 v = ml[s];
    if (v.y != 0.f) M = fmaxf(M, v.x);
  }
  M = wave_max(M);
  if (tid % kWave == 0) s_red[tid / kWave] = M;
  __syncthreads();
  M = s_red[0];
#pragma unroll
  for (int w = 1; w < kJoinThreads / kWave; ++w) M = fmaxf(M, s_red[w]);
  __syncthreads();
  float sum = 0.f;
  for (int s = tid; s < runs; s += kJoinThreads) {
    const float2 v = ml[s];
    const float f = v.y != 0.f ? exp2f(v.x - M) : 0.f;
    s_f[s] = f;
    sum = v.y != 0.f ? fmaf(v.y, f, sum) : sum;
  }
  sum = wave_sum(sum);
  if (tid % kWave == 0) s_red[tid / kWave] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinThreads / kWave; ++w) sum += s_red[w];

  const int r = tid / kLanes, c = tid % kLanes;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (r < kRows) {
    const f32x4* o = reinterpret_cast<const f32x4*>(part_o + row * runs * D) + c;
    for (int s = r; s < runs; s += kRows) acc += o[int64_t(s) * kLanes] * s_f[s];
    s_acc[r][c] = acc;
  }
  __syncthreads();
  if (r != 0) return;
#pragma unroll
  for (int i = 1; i < kRows; ++i) acc += s_acc[i][c];
  const float k = sum == 0.f ? 0.f : (p.v_scale ? p.v_scale[row % p.hq / (p.hq / p.hk)] : 1.f) / sum;
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = sum == 0.f ? 0u : pack2<T>(acc[2 * i] * k, acc[2 * i + 1] * k);
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + row * D + c * 4) = w;
  if (p.lse && c == 0) p.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

// How the tokens of the longest sequence are cut: about four blocks a compute
// unit over the whole call, and at least two tiles a wave.
struct Plan {
  int tiles_per_run, runs;
};
Plan plan(int64_t batch, int64_t hq, int64_t hk, int64_t span) {
  const int64_t tiles = (span + kTile - 1) / kTile;
  const int64_t blocks = batch * hk * ((hq / hk + 15) / 16);
  const int64_t want = std::max<int64_t>(1, (1024 + blocks - 1) / blocks);
  const int64_t least = 2 * kWaves;
  int64_t per = std::max(least, (tiles + want - 1) / want);
  per = (per + kWaves - 1) / kWaves * kWaves;
  return {int(per), int(std::max<int64_t>(1, (tiles + per - 1) / per))};
}

// Tokens from the first one's tile on that a sequence can span.
int64_t span_of(int64_t max_length, int64_t window) {
  return window > 0 && window + kTile < max_length ? window + kTile : max_length;
}

template <class T, bool C8, int D>
hipError_t launch(const AttendParams& p, hipStream_t stream) {
  const Plan c = plan(p.batch, p.hq, p.hk, span_of(p.max_length, p.window));
  const int64_t rows = int64_t(p.batch) * p.hq;
  float* part_ml = static_cast<float*>(p.workspace);
  float* part_o = part_ml + (rows * c.runs * 2 + 63) / 64 * 64;
  const dim3 grid(unsigned(c.runs), unsigned(p.hk * ((p.hq / p.hk + 15) / 16)), unsigned(p.batch));
  attend_kernel<T, C8, D><<<grid, dim3(64 * kWaves), 0, stream>>>(p, c.tiles_per_run, c.runs, part_o, part_ml);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.runs == 1) return e;
  attend_join_kernel<T, D><<<dim3(unsigned(rows)), dim3(kJoinThreads), c.runs * sizeof(float), stream>>>(p, c.runs, part_o, part_ml);
  return hipGetLastError();
}

template <class T, bool C8>
hipError_t launch_dim(const AttendParams& p, hipStream_t stream) {
  switch (p.d) {
    case 64: return launch<T, C8, 64>(p, stream);
    case 96: return launch<T, C8, 96>(p, stream);
    case 128: return launch<T, C8, 128>(p, stream);
    case 192: return launch<T, C8, 192>(p, stream);
    case 256: return launch<T, C8, 256>(p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace

size_t attend_workspace_bytes(int64_t batch, int64_t hq, int64_t hk, int64_t d, int64_t max_length, int64_t window) {
  const Plan c = plan(batch, hq, hk, span_of(max_length, window));
  if (c.runs == 1) return 0;
  const int64_t rows = batch * hq;
  return size_t((rows * c.runs * 2 + 63) / 64 * 64 + rows * c.runs * d) * sizeof(float);
}

hipError_t launch_attend(const AttendParams& p, hipStream_t stream) {
  if (p.type == ServeType::kBf16) return p.cache8 ? launch_dim<Bf16, true>(p, stream) : launch_dim<Bf16, false>(p, stream);
  return p.cache8 ? launch_dim<F16, true>(p, stream) : launch_dim<F16, false>(p, stream);
}

}  // namespace cp
