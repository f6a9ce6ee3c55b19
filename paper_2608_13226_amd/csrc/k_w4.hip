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
// A wave works on 16 outputs (the rows of A) and MT times 16 rows of x (the
// columns of B); the block's waves share the outputs and take runs of 128 k
// in turn, and their sums meet in LDS.  A lane loads 16 bytes of one output's
// codes, 32 k: where groups are multiples of 128 that is how the products take
// them (lane group g holds k = 32 g + 8 j at step j); smaller groups need each
// step's 32 k from one group, so the four lane groups exchange their words
// first (k = 32 j + 8 g).
#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

constexpr int kWaves = 4;

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
template <class T, bool X8>
__device__ __forceinline__ u32x4 load_x(const void* x, int64_t i) {
  if constexpr (X8) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(x) + i);
    const uint32_t even = __builtin_amdgcn_perm(w[1], w[0], 0x06040200u), odd = __builtin_amdgcn_perm(w[1], w[0], 0x07050301u);
    return u32x4{widen2<T, false>(even), widen2<T, true>(even), widen2<T, false>(odd), widen2<T, true>(odd)};
  } else {
    return order<T>(*reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(x) + i));
  }
}

template <class T>
__device__ __forceinline__ uint32_t one2() { return pack2<T>(1.f, 1.f); }

template <class T, bool X8, bool SMALL, int MT>
__global__ __launch_bounds__(64 * kWaves) void w4_kernel(W4Params p) {
  __shared__ float s_part[kWaves][MT][16][17];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane % 16, g = lane / 16;
  const int64_t n0 = int64_t(blockIdx.x) * 16, m0 = int64_t(blockIdx.y) * (16 * MT);
  const int groups = p.k / p.group;
  const int64_t row = n0 + c < p.n ? n0 + c : p.n - 1;
  const uint8_t* wrow = p.weight + row * (p.k / 2);
  const u32x4 ones = {one2<T>(), one2<T>(), one2<T>(), one2<T>()};
  f32x4 y[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) y[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int kb = wave * 128; kb < p.k; kb += kWaves * 128) {
    uint32_t w[4] = {0, 0, 0, 0};
    if (kb + g * 32 < p.k) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(wrow + (kb + g * 32) / 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = v[j];
    }
    if constexpr (SMALL) transpose4(w);
    f32x4 acc[MT], sum[MT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (SMALL && kb + j * 32 >= p.k) break;
      if (SMALL || j == 0) {
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      const u32x4 a = codes<T>(w[j]);
      const int k = kb + (SMALL ? j * 32 + g * 8 : g * 32 + j * 8);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int64_t i = m0 + t * 16 + c;
        u32x4 b = {0, 0, 0, 0};
        if (i < p.m) b = load_x<T, X8>(p.x, i * p.k + k);
        acc[t] = mfma32<T>(a, b, acc[t]);
        sum[t] = mfma32<T>(ones, b, sum[t]);
      }
      if (SMALL || j == 3) {
        const int group = (kb + (SMALL ? j * 32 : 0)) / p.group;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t nr = n0 + g * 4 + r < p.n ? n0 + g * 4 + r : p.n - 1;
          const float s = load1<T>(p.scale, nr * groups + group);
          const float z = p.zero ? float(p.zero[nr * groups + group]) : 8.f;
#pragma unroll
          for (int t = 0; t < MT; ++t) y[t][r] = fmaf(s, fmaf(512.f, acc[t][r], -z * sum[t][r]), y[t][r]);
        }
      }
    }
  }

#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) s_part[wave][t][c][g * 4 + r] = y[t][r];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += 64 * kWaves) {
    const int t = i / 256, mr = (i / 16) % 16, nr = i % 16;
    const int64_t m = m0 + t * 16 + mr, n = n0 + nr;
    if (m >= p.m || n >= p.n) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += s_part[w][t][mr][nr];
    if (X8) v *= p.x_scale[m];
    if (p.y_type == ServeType::kF32) store1<F32>(p.y, m * p.n + n, v);
    else store1<T>(p.y, m * p.n + n, v);
  }
}

template <class T, bool X8, bool SMALL, int MT>
hipError_t launch(const W4Params& p, hipStream_t stream) {
  const dim3 grid(unsigned((p.n + 15) / 16), unsigned((p.m + 16 * MT - 1) / (16 * MT)));
  w4_kernel<T, X8, SMALL, MT><<<grid, dim3(64 * kWaves), 0, stream>>>(p);
  return hipGetLastError();
}

template <class T, bool X8>
hipError_t launch_type(const W4Params& p, hipStream_t stream) {
  const bool small = p.group % 128 != 0;
  if (p.m <= 16) return small ? launch<T, X8, true, 1>(p, stream) : launch<T, X8, false, 1>(p, stream);
  return small ? launch<T, X8, true, 4>(p, stream) : launch<T, X8, false, 4>(p, stream);
}

}  // namespace

hipError_t launch_w4_matvec(const W4Params& p, hipStream_t stream) {
  if (p.type == ServeType::kBf16) return p.x_scale ? launch_type<Bf16, true>(p, stream) : launch_type<Bf16, false>(p, stream);
  return p.x_scale ? launch_type<F16, true>(p, stream) : launch_type<F16, false>(p, stream);
}

}  // namespace cp
