// Root-mean-square norm with the residual's addition, rounded to the input's
// type or to e4m3 with a scale per row:
//   h = x + r,  y_j = h_j w_j / sqrt(mean_j h_j^2 + eps),
//   scale = max_j |y_j| / 448,  code_j = e4m3(y_j / scale).
//
// Bound by memory: each row is read once and held in registers in float32
// between the sum of squares and the outputs, so the norm is of the unrounded
// h and the residual stream is rounded once.  A block works on one row, a
// thread has every blockDim.x-th run of eight elements: 6272 rows of 3584 to
// e4m3 in 34.3 us (4.6 TB/s).  (A wave a row without barriers, and two or four
// rows a block, measured no better: 39 us, 39 and 52 where this took 36.1.)
#include <type_traits>

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

// Eight elements from i on, of which `left` are the row's.  ANY: d is no
// multiple of 8, so rows begin anywhere and their last run is short; zeros
// stand for what it lacks.  The hardware takes wide accesses at any address
// (5437 rows of 3091, bf16: 19.9 us, element by element 35.4).
constexpr int kRun = 8;
template <class T, bool ANY>
__device__ __forceinline__ void load_run(const void* p, int64_t i, int left, float* x) {
  if constexpr (!ANY) {
    load8<T>(p, i, x);
  } else if (left >= kRun) {
    using Element = std::conditional_t<std::is_same_v<T, F32>, float, uint16_t>;
    alignas(16) Element w[kRun];
    __builtin_memcpy(w, static_cast<const Element*>(p) + i, sizeof w);
    load8<T>(w, 0, x);
  } else {
#pragma unroll
    for (int e = 0; e < kRun; ++e) x[e] = e < left ? load1<T>(p, i + e) : 0.f;
  }
}
template <class T, bool ANY>
__device__ __forceinline__ void store_run(void* p, int64_t i, int left, const float* x) {
  if constexpr (!ANY) {
    store8<T>(p, i, x);
  } else if (left >= kRun) {
    using Element = std::conditional_t<std::is_same_v<T, F32>, float, std::conditional_t<std::is_same_v<T, E4m3>, uint8_t, uint16_t>>;
    alignas(16) Element w[kRun];
    store8<T>(w, 0, x);
    __builtin_memcpy(static_cast<Element*>(p) + i, w, sizeof w);
  } else {
#pragma unroll
    for (int e = 0; e < kRun; ++e)
      if (e < left) store1<T>(p, i + e, x[e]);
  }
}

template <class T, bool Q, bool ANY, int NV>
__global__ __launch_bounds__(1024) void rms_norm_kernel(RmsNormParams p, int64_t first) {
  __shared__ float s_sum[4][16];
  __shared__ unsigned s_top[4][16];
  const int64_t row = first + blockIdx.x;
  const int64_t base = row * p.d;
  float h[NV][kRun];
  float sq = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
    if (j < p.d) load_run<T, ANY>(p.x, base + j, p.d - j, h[v]);
  }
  if (p.residual) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
      if (j < p.d) {
        float r[kRun];
        load_run<T, ANY>(p.residual, base + j, p.d - j, r);
#pragma unroll
        for (int e = 0; e < kRun; ++e) h[v][e] += r[e];
        store_run<T, ANY>(p.residual_out, base + j, p.d - j, h[v]);
      }
    }
  }
  // With 8 bits the largest |h w| is found in the same pass: the row's factor
  // 1 / rms cancels from the codes.
  unsigned top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
    if (j < p.d) {
      float w[kRun];
      if constexpr (Q) load_run<T, ANY>(p.weight, j, p.d - j, w);
#pragma unroll
      for (int e = 0; e < kRun; ++e) {
        sq = fmaf(h[v][e], h[v][e], sq);
        if constexpr (Q) top = max(top, __float_as_uint(fabsf(h[v][e] * w[e])));
      }
    }
  }
  row_reduce(sq, top, s_sum[0], s_top[0]);
  float rms = 1.f / sqrtf(sq / float(p.d) + p.eps);
  if (!(sq > 1e-25f && sq < 1e37f)) {
    // Squares at the ends of float32's range: the same with h over a power of
    // two near its largest.  (Nothing changes for zeros, infinities and NaN,
    // nor where eps is so large beside the squares that they do not count:
    // their sum over the power's square is below 2^18.)
    float scaled = 0.f;
    unsigned most = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if ((v * int(blockDim.x) + int(threadIdx.x)) * kRun < p.d)
#pragma unroll
        for (int e = 0; e < kRun; ++e) most = max(most, __float_as_uint(fabsf(h[v][e])));
    row_reduce(scaled, most, s_sum[1], s_top[1]);
    if (most > 0 && most < 0x7f800000u) {
      const int exponent = max(int(most >> 23), 1) - 127;
      const float s = ldexpf(1.f, -exponent);
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if ((v * int(blockDim.x) + int(threadIdx.x)) * kRun < p.d)
#pragma unroll
          for (int e = 0; e < kRun; ++e) scaled = fmaf(h[v][e] * s, h[v][e] * s, scaled);
      row_reduce(scaled, most, s_sum[2], s_top[2]);
      const float eps = p.eps * s * s;
      if (eps < 1e30f) {
        const float root = sqrtf(scaled / float(p.d) + eps);
        rms = s / root;
        if (rms > 3.4e38f) {
          // 1 / rms itself is past float32: h over the power takes h's place, and
          // 8 bits go step by step.
          rms = 1.f / root;
          top = 0;
#pragma unroll
          for (int v = 0; v < NV; ++v)
            if ((v * int(blockDim.x) + int(threadIdx.x)) * kRun < p.d)
#pragma unroll
              for (int e = 0; e < kRun; ++e) h[v][e] *= s;
        }
      }
    }
  }
  if constexpr (!Q) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
      if (j < p.d) {
        float w[kRun];
        load_run<T, ANY>(p.weight, j, p.d - j, w);
#pragma unroll
        for (int e = 0; e < kRun; ++e) h[v][e] = h[v][e] * rms * w[e];
        store_run<T, ANY>(p.out, base + j, p.d - j, h[v]);
      }
    }
  } else {
    const float most = __uint_as_float(top);
    float scale = most * rms / kE4m3Max;
    if (most > 1e-30f && most < 1e30f && scale > 1e-30f) {
      // One division a row, whose quotient is kept in two parts so that a code is
      // that of h w / (most / 448) to float32's last bit; no product passes 448 by
      // more than float32's rounding.
      const float factor = kE4m3Max / most, rest = fmaf(-factor, most, kE4m3Max) / most;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
        if (j < p.d) {
          float w[kRun];
          load_run<T, ANY>(p.weight, j, p.d - j, w);
#pragma unroll
          for (int e = 0; e < kRun; ++e) {
            const float y = h[v][e] * w[e];
            h[v][e] = fmaf(y, factor, y * rest);
          }
          uint8_t* out = static_cast<uint8_t*>(p.out) + base + j;
          const u32x2 codes = {pack4_e4m3_inside(h[v][0], h[v][1], h[v][2], h[v][3]),
                               pack4_e4m3_inside(h[v][4], h[v][5], h[v][6], h[v][7])};
          if (!ANY) *reinterpret_cast<u32x2*>(out) = codes;
          else if (p.d - j >= kRun) __builtin_memcpy(out, &codes, sizeof codes);
          else
#pragma unroll
            for (int e = 0; e < kRun - 1; ++e)
              if (e < p.d - j) out[e] = uint8_t(codes[e / 4] >> e % 4 * 8);
        }
      }
    } else {
      // Zeros, NaN, infinities and products near the ends of float32's range:
      // as the formula says, step by step.
      top = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
        if (j < p.d) {
          float w[kRun];
          load_run<T, ANY>(p.weight, j, p.d - j, w);
#pragma unroll
          for (int e = 0; e < kRun; ++e) {
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
        const int j = (v * int(blockDim.x) + int(threadIdx.x)) * kRun;
        if (j < p.d) {
#pragma unroll
          for (int e = 0; e < kRun; ++e) h[v][e] = scale == 0.f ? 0.f : h[v][e] / scale;
          store_run<E4m3, ANY>(p.out, base + j, p.d - j, h[v]);
        }
      }
    }
    if (threadIdx.x == 0) p.out_scale[row] = scale;
  }
}

template <class T, bool Q, bool ANY>
hipError_t launch(const RmsNormParams& p, hipStream_t stream) {
  const int runs = (p.d + kRun - 1) / kRun;
  const int threads = runs >= 1024 ? 1024 : (runs + kWave - 1) / kWave * kWave;
  const int nv = (runs + threads - 1) / threads;
  return launch_blocks(p.rows, threads, [&](int64_t first, unsigned rows) {
    const dim3 grid(rows), block(threads);
    if (nv <= 1) rms_norm_kernel<T, Q, ANY, 1><<<grid, block, 0, stream>>>(p, first);
    else if (nv <= 2) rms_norm_kernel<T, Q, ANY, 2><<<grid, block, 0, stream>>>(p, first);
    else if (nv <= 4) rms_norm_kernel<T, Q, ANY, 4><<<grid, block, 0, stream>>>(p, first);
    else rms_norm_kernel<T, Q, ANY, 8><<<grid, block, 0, stream>>>(p, first);
  });
}

template <class T, bool Q>
hipError_t launch_type(const RmsNormParams& p, hipStream_t stream) {
  return p.d % kRun == 0 ? launch<T, Q, false>(p, stream) : launch<T, Q, true>(p, stream);
}

}  // namespace

hipError_t launch_rms_norm(const RmsNormParams& p, hipStream_t stream) {
  if (p.type == ServeType::kBf16) return p.quantize ? launch_type<Bf16, true>(p, stream) : launch_type<Bf16, false>(p, stream);
  if (p.type == ServeType::kF16) return p.quantize ? launch_type<F16, true>(p, stream) : launch_type<F16, false>(p, stream);
  return p.quantize ? launch_type<F32, true>(p, stream) : launch_type<F32, false>(p, stream);
}

}  // namespace cp
