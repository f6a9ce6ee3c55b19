// Root-mean-square norm with the residual's addition, rounded to the input's
// type or to e4m3 with a scale per row:
//   h = x + r,  y_j = h_j w_j / sqrt(mean_j h_j^2 + eps),
//   scale = max_j |y_j| / 448,  code_j = e4m3(y_j / scale).
//
// Bound by memory: each row is read once and held in registers in float32
// between the sum of squares and the outputs, so the norm is of the unrounded
// h and the residual stream is rounded once.  A block works on one row, a
// thread has every blockDim.x-th run of VEC elements.  (A wave a row without
// barriers, and two or four rows a block, measured no better: 6272 rows of
// 3584 to e4m3 36.1 us, 39, 39 and 52.)
#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// Sum of x and maximum of m over the block, whose threads all get them.  m: bits
// of values >= 0, which order like the values; a NaN's are above all others',
// so it stays.
__device__ __forceinline__ void row_reduce(float& x, unsigned& m, float* s, unsigned* t) {
  x = wave_sum(x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, unsigned(__shfl_xor(int(m), o)));
  const int waves = blockDim.x / kWave;
  if (waves == 1) return;
  if (threadIdx.x % kWave == 0) {
    s[threadIdx.x / kWave] = x;
    t[threadIdx.x / kWave] = m;
  }
  __syncthreads();
  x = 0.f;
  m = 0;
  for (int i = 0; i < waves; ++i) {
    x += s[i];
    m = max(m, t[i]);
  }
}

template <class T, int VEC>
__device__ __forceinline__ void load_run(const void* p, int64_t i, float* x) {
  if constexpr (VEC == 8) load8<T>(p, i, x);
  else x[0] = load1<T>(p, i);
}
template <class T, int VEC>
__device__ __forceinline__ void store_run(void* p, int64_t i, const float* x) {
  if constexpr (VEC == 8) store8<T>(p, i, x);
  else store1<T>(p, i, x[0]);
}

template <class T, bool Q, int VEC, int NV>
__global__ __launch_bounds__(1024) void rms_norm_kernel(RmsNormParams p) {
  __shared__ float s_sum[4][16];
  __shared__ unsigned s_top[4][16];
  const int64_t row = blockIdx.x;
  const int64_t base = row * p.d;
  float h[NV][VEC];
  float sq = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
    if (j < p.d) load_run<T, VEC>(p.x, base + j, h[v]);
  }
  if (p.residual) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
      if (j < p.d) {
        float r[VEC];
        load_run<T, VEC>(p.residual, base + j, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[v][e] += r[e];
        store_run<T, VEC>(p.residual_out, base + j, h[v]);
      }
    }
  }
  // With 8 bits the largest |h w| is found in the same pass: the row's factor
  // 1 / rms cancels from the codes.
  unsigned top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
    if (j < p.d) {
      float w[VEC];
      if constexpr (Q) load_run<T, VEC>(p.weight, j, w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        sq = fmaf(h[v][e], h[v][e], sq);
        if constexpr (Q) top = max(top, __float_as_uint(fabsf(h[v][e] * w[e])));
      }
    }
  }
  row_reduce(sq, top, s_sum[0], s_top[0]);
  float rms = 1.f / sqrtf(sq / float(p.d) + p.eps);
  if (!(sq > 1e-25f && sq < 1e37f)) {
    // Squares at the ends of float32's range: the same with h over a power of
    // two near its largest.  (Nothing changes for zeros, infinities and NaN.)
    float scaled = 0.f;
    unsigned most = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if ((v * int(blockDim.x) + int(threadIdx.x)) * VEC < p.d)
#pragma unroll
        for (int e = 0; e < VEC; ++e) most = max(most, __float_as_uint(fabsf(h[v][e])));
    row_reduce(scaled, most, s_sum[1], s_top[1]);
    if (most > 0 && most < 0x7f800000u) {
      const int exponent = max(int(most >> 23), 1) - 127;
      const float s = ldexpf(1.f, -exponent);
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if ((v * int(blockDim.x) + int(threadIdx.x)) * VEC < p.d)
#pragma unroll
          for (int e = 0; e < VEC; ++e) scaled = fmaf(h[v][e] * s, h[v][e] * s, scaled);
      row_reduce(scaled, most, s_sum[2], s_top[2]);
      rms = s / sqrtf(scaled / float(p.d) + p.eps * s * s);
    }
  }
  if constexpr (!Q) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
      if (j < p.d) {
        float w[VEC];
        load_run<T, VEC>(p.weight, j, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[v][e] = h[v][e] * rms * w[e];
        store_run<T, VEC>(p.out, base + j, h[v]);
      }
    }
  } else {
    const float most = __uint_as_float(top);
    float scale = most * rms / kE4m3Max;
    if (most > 1e-30f && most < 1e30f && scale > 1e-30f) {
      // One division a row; no product passes 448 by more than float32's rounding.
      const float factor = kE4m3Max / most;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
        if (j < p.d) {
          float w[VEC];
          load_run<T, VEC>(p.weight, j, w);
#pragma unroll
          for (int e = 0; e < VEC; ++e) h[v][e] = h[v][e] * w[e] * factor;
          uint8_t* out = static_cast<uint8_t*>(p.out) + base + j;
          if constexpr (VEC == 8)
            *reinterpret_cast<u32x2*>(out) = u32x2{pack4_e4m3_inside(h[v][0], h[v][1], h[v][2], h[v][3]),
                                                   pack4_e4m3_inside(h[v][4], h[v][5], h[v][6], h[v][7])};
          else
            *out = uint8_t(pack4_e4m3_inside(h[v][0], 0.f, 0.f, 0.f));
        }
      }
    } else {
      // Zeros, NaN, infinities and products near the ends of float32's range:
      // as the formula says, step by step.
      top = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
        if (j < p.d) {
          float w[VEC];
          load_run<T, VEC>(p.weight, j, w);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            h[v][e] = h[v][e] * rms * w[e];
            top = max(top, __float_as_uint(fabsf(h[v][e])));
          }
        }
      }
      float unused = 0.f;
      row_reduce(unused, top, s_sum[3], s_top[3]);
      scale = __uint_as_float(top) / kE4m3Max;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
        if (j < p.d) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) h[v][e] = scale == 0.f ? 0.f : h[v][e] / scale;
          store_run<E4m3, VEC>(p.out, base + j, h[v]);
        }
      }
    }
    if (threadIdx.x == 0) p.out_scale[row] = scale;
  }
}

template <class T, bool Q, int VEC, int NV>
hipError_t launch(const RmsNormParams& p, int threads, hipStream_t stream) {
  rms_norm_kernel<T, Q, VEC, NV><<<dim3(unsigned(p.rows)), dim3(threads), 0, stream>>>(p);
  return hipGetLastError();
}

template <class T, bool Q>
hipError_t launch_type(const RmsNormParams& p, hipStream_t stream) {
  const int vec = p.d % 8 == 0 ? 8 : 1;
  const int runs = (p.d + vec - 1) / vec;
  const int threads = runs >= 1024 ? 1024 : (runs + kWave - 1) / kWave * kWave;
  const int nv = (runs + threads - 1) / threads;
  if (vec == 8) {
    if (nv <= 1) return launch<T, Q, 8, 1>(p, threads, stream);
    if (nv <= 2) return launch<T, Q, 8, 2>(p, threads, stream);
    if (nv <= 4) return launch<T, Q, 8, 4>(p, threads, stream);
    return launch<T, Q, 8, 8>(p, threads, stream);
  }
  if (nv <= 8) return launch<T, Q, 1, 8>(p, threads, stream);
  return launch<T, Q, 1, 64>(p, threads, stream);
}

}  // namespace

hipError_t launch_rms_norm(const RmsNormParams& p, hipStream_t stream) {
  if (p.type == ServeType::kBf16) return p.quantize ? launch_type<Bf16, true>(p, stream) : launch_type<Bf16, false>(p, stream);
  if (p.type == ServeType::kF16) return p.quantize ? launch_type<F16, true>(p, stream) : launch_type<F16, false>(p, stream);
  return p.quantize ? launch_type<F32, true>(p, stream) : launch_type<F32, false>(p, stream);
}

}  // namespace cp
