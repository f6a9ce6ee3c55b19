// Root-mean-square norm with the residual's addition, rounded to the input's
// type or to e4m3 with a scale per row:
//   h = x + r,  y_j = h_j w_j / sqrt(mean_j h_j^2 + eps),
//   scale = max_j |y_j| / 448,  code_j = e4m3(y_j / scale).
//
// Bound by memory: each row is read once and held in registers in float32
// between the sum of squares and the outputs, so the norm is of the unrounded
// h and the residual stream is rounded once.  A block works on one row, a
// thread on every blockDim.x-th run of VEC elements.
#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// Sum over the block; every thread gets it.
__device__ __forceinline__ float block_sum(float x, float* s) {
  x = wave_sum(x);
  const int waves = blockDim.x / kWave;
  if (waves == 1) return x;
  if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = x;
  __syncthreads();
  float t = 0.f;
  for (int i = 0; i < waves; ++i) t += s[i];
  return t;
}
// Maximum over the block of bits of values >= 0, which order like the values;
// a NaN's are above all others', so it stays.
__device__ __forceinline__ unsigned block_max(unsigned x, unsigned* s) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, unsigned(__shfl_xor(int(x), o)));
  const int waves = blockDim.x / kWave;
  if (waves == 1) return x;
  if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = x;
  __syncthreads();
  unsigned t = 0;
  for (int i = 0; i < waves; ++i) t = max(t, s[i]);
  return t;
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
  __shared__ float s_sum[16];
  __shared__ unsigned s_max[16];
  const int64_t row = blockIdx.x;
  const int64_t base = row * p.d;
  float h[NV][VEC];
  float sq = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
    if (j < p.d) {
      load_run<T, VEC>(p.x, base + j, h[v]);
      if (p.residual) {
        float r[VEC];
        load_run<T, VEC>(p.residual, base + j, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[v][e] += r[e];
        store_run<T, VEC>(p.residual_out, base + j, h[v]);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sq = fmaf(h[v][e], h[v][e], sq);
    }
  }
  const float rms = 1.f / sqrtf(block_sum(sq, s_sum) / float(p.d) + p.eps);
  unsigned top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
    if (j < p.d) {
      float w[VEC];
      load_run<T, VEC>(p.weight, j, w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        h[v][e] = h[v][e] * rms * w[e];
        if constexpr (Q) top = max(top, __float_as_uint(fabsf(h[v][e])));
      }
      if constexpr (!Q) store_run<T, VEC>(p.out, base + j, h[v]);
    }
  }
  if constexpr (Q) {
    const float scale = __uint_as_float(block_max(top, s_max)) / kE4m3Max;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int j = (v * int(blockDim.x) + int(threadIdx.x)) * VEC;
      if (j < p.d) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[v][e] = scale == 0.f ? 0.f : h[v][e] / scale;
        store_run<E4m3, VEC>(p.out, base + j, h[v]);
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
