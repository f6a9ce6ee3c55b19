// Position rotation of queries and keys, and keys and values into a paged cache
// of 4 bits, in one pass.
//
// A block of 32 elements x is held as s = 2^e, the smallest power (of those
// whose values are normal and finite in T) with max |x| <= 6 s, and the codes
// of x / s rounded to nearest, ties to the even code; what lies beyond 6 s of the
// largest power becomes that.  Bound by memory: every element is read once and
// written once, queries in 16 bits, keys and values in 4.25.
//
// Codes are those of the key rotated in float64: a float32 rotation would put
// one code in 10^6 on the other side of a border.  The angle, position *
// inv_freq, is reduced to a fraction of a turn with 1 / 2 pi in two parts, so that
// it is off by the rounding of the product alone.  A key goes to float32 rounded to
// odd (towards zero, last bit set where something was cut), which keeps it on
// its side of every border.  Queries are rotated in float32, as in kv_append.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// float64 to float32, rounded to odd: of the 29 bits that go, whether any was set stays in the
// last one of the others, and the conversion is exact.  (Past float32's range: infinite.)
__device__ __forceinline__ float round_odd(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t low = uint32_t(b), kept = (low & 0xe0000000u) | (low & 0x1fffffffu ? 0x20000000u : 0u);
  return float(__builtin_bit_cast(double, (b & 0xffffffff00000000u) | kept));
}

// Eight elements from element i on.
template <class T, bool WIDE>
__device__ __forceinline__ void load_run(const void* p, int64_t i, float* x) {
  if constexpr (WIDE) {
    load8<T>(p, i, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = load1<T>(p, i + j);
  }
}

// The exponents that a block may have, plus 127.
template <class T> constexpr int kLeast = 2;
template <class T> constexpr int kMost = 252;
template <> constexpr int kLeast<F16> = 104;
template <> constexpr int kMost<F16> = 140;

// Four neighbouring lanes' eight elements each as a block: this lane's codes, and the exponent byte.
template <class T>
__device__ __forceinline__ uint32_t cut_block(const float* x, uint32_t* exponent) {
  // As whole numbers the bits of |x| are in its order, infinities and NaN last.
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0xb1, 0xf, 0xf, true)));     // lane ^ 1
  top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0x4e, 0xf, 0xf, true)));     // lane ^ 2
  if (top >= 0x7f800000u) {
    *exponent = 255u;
    return 0u;
  }
  // 6 * 2^e = 1.5 * 2^(e + 2).
  const int e = int(top >> 23) - 1 - ((top & 0x7fffffu) <= 0x400000u ? 1 : 0);
  *exponent = uint32_t(min(max(e, kLeast<T>), kMost<T>));
  const float s = power_of(*exponent);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return w;
}

// The run's elements e + 0..7 of a head whose first is element `head` of p, turned:
// `own` holds them, cosines and sines of the pairs are cs[pair].  R: float or double.
template <class T, bool INTER, bool WIDE, class R>
__device__ __forceinline__ void turn_run(const void* p, int64_t head, int e, int rot, const R* cosines, const R* sines,
                                         const float* own, R* y) {
  const int half = rot / 2;
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = own[j];
  if (e >= rot) return;
  if constexpr (INTER) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      if (e + j >= rot) break;
      const R c = cosines[(e + j) / 2], s = sines[(e + j) / 2], a = own[j], b = own[j + 1];
      y[j] = a * c - b * s;
      y[j + 1] = b * c + a * s;
    }
  } else if (WIDE && half % 8 == 0) {
    const bool second = e >= half;
    const int i0 = second ? e - half : e;
    float other[8];
    load_run<T, true>(p, head + (second ? i0 : e + half), other);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const R c = cosines[i0 + j], s = sines[i0 + j], a = own[j], b = other[j];
      y[j] = second ? a * c + b * s : a * c - b * s;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (e + j >= rot) break;
      const bool second = e + j >= half;
      const int i = second ? e + j - half : e + j;
      const R c = cosines[i], s = sines[i], a = own[j], b = load1<T>(p, head + (second ? i : i + half));
      y[j] = second ? a * c + b * s : a * c - b * s;
    }
  }
}

// A block of 256 has `threads` for each of its tokens; a thread has runs of eight
// elements, queries' first, then keys', then values'.  WIDE: rows are 16-byte aligned.
template <class T, bool INTER, bool WIDE>
__global__ __launch_bounds__(256) void kv_append4_kernel(KvAppend4Params p, int threads, int64_t first_block) {
  extern __shared__ double s_turns[];         // a token's [rot / 2] cosines, sines, and both again as floats
  const int tid = threadIdx.x % threads, mine = threadIdx.x / threads;
  const int64_t token = (first_block + blockIdx.x) * (256 / threads) + mine, t = min(token, p.tokens - 1);
  const int half = p.rot / 2;
  double *s_cos = s_turns + int64_t(mine) * half * 3, *s_sin = s_cos + half;
  float *s_cosf = reinterpret_cast<float*>(s_sin + half), *s_sinf = s_cosf + half;
  const double position = double(p.positions[t]);
  const int64_t slot = p.slots[t];
  const bool here = token < p.tokens, keep = here && slot >= 0 && slot < p.pages * p.page;
  for (int i = tid; i < half; i += threads) {
    const double angle = position * double(p.inv_freq[i]);
    // angle / 2 pi less its whole turns; 1 / 2 pi = high + low.
    const double high = 0.15915494309189535, low = -9.839338337591243e-18;
    const double turns = angle * high, rest = fma(angle, high, -turns) + angle * low;
    double s, c;
    sincospi(2.0 * ((turns - rint(turns)) + rest), &s, &c);
    c *= double(p.magnitude);
    s *= double(p.magnitude);
    s_cos[i] = c;
    s_sin[i] = s;
    s_cosf[i] = float(c);
    s_sinf[i] = float(s);
  }
  __syncthreads();
  if (!here) return;
  const int runs = p.d / 8, hq = p.q ? p.hq : 0;
  const int64_t pg = keep ? page_of(slot, p.page, p.by_page) : 0, off = keep ? slot - pg * p.page : 0;
  const int total = (hq + (keep ? 2 * p.hk : 0)) * runs;
  for (int w = int(blockIdx.y) * threads + tid; w < total; w += int(gridDim.y) * threads) {
    const int head = int(p.by_runs(unsigned(w))), e = (w - head * runs) * 8;
    if (head < hq) {
      const int64_t from = t * p.q_stride + int64_t(head) * p.d;
      float x[8], y[8];
      load_run<T, WIDE>(p.q, from + e, x);
      turn_run<T, INTER, WIDE, float>(p.q, from, e, p.rot, s_cosf, s_sinf, x, y);
      store8<T>(p.q_out, (t * p.hq + head) * p.d + e, y);
      continue;
    }
    const bool is_k = head < hq + p.hk;
    const int kh = head - hq - (is_k ? 0 : p.hk);
    const void* src = is_k ? p.k : p.v;
    const int64_t from = t * (is_k ? p.k_stride : p.v_stride) + int64_t(kh) * p.d;
    float x[8];
    load_run<T, WIDE>(src, from + e, x);
    if (is_k) {
      double y[8];
      turn_run<T, INTER, WIDE, double>(src, from, e, p.rot, s_cos, s_sin, x, y);
      if (e < p.rot) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = round_odd(y[j]);
        // What is finite but past float32's range counts as its largest number.
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));
        if (most > 3e38f) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (fabs(y[j]) < __builtin_inf()) x[j] = float(fmin(fmax(y[j], -3.4028234663852886e38), 3.4028234663852886e38));
        }
      }
    }
    uint32_t exponent;
    const uint32_t codes = cut_block<T>(x, &exponent);
    const int64_t row = (pg * p.hk + kh) * p.page + off;
    *reinterpret_cast<uint32_t*>((is_k ? p.k_cache : p.v_cache) + row * (p.d / 2) + e / 2) = codes;
    if (e % kBlock4 == 0) (is_k ? p.k_scale : p.v_scale)[row * (p.d / kBlock4) + e / kBlock4] = uint8_t(exponent);
  }
}

template <class T, bool INTER, bool WIDE>
hipError_t launch(const KvAppend4Params& p, hipStream_t stream) {
  const int64_t work = (int64_t(p.q ? p.hq : 0) + 2 * p.hk) * (p.d / 8);
  const unsigned y = unsigned(std::max<int64_t>(1, std::min<int64_t>(2048 / p.tokens, (work + 255) / 256)));
  int threads = 256;
  while (threads > 32 && threads / 2 >= work / 4 && p.tokens * (threads / 2) >= 256 * 256) threads /= 2;
  const int64_t per = 256 / threads;
  return launch_blocks((p.tokens + per - 1) / per, 256, [&](int64_t first, unsigned blocks) {
    kv_append4_kernel<T, INTER, WIDE><<<dim3(blocks, y), dim3(256), size_t(per) * p.rot * 12, stream>>>(p, threads, first);
  });
}

bool aligned(const void* q, int64_t stride) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && stride % 8 == 0; }

template <class T>
hipError_t launch_type(const KvAppend4Params& p, hipStream_t stream) {
  const bool wide = (!p.q || aligned(p.q, p.q_stride)) && aligned(p.k, p.k_stride) && aligned(p.v, p.v_stride);
  if (p.interleaved) return wide ? launch<T, true, true>(p, stream) : launch<T, true, false>(p, stream);
  return wide ? launch<T, false, true>(p, stream) : launch<T, false, false>(p, stream);
}

}  // namespace

hipError_t launch_kv_append4(const KvAppend4Params& p, hipStream_t stream) {
  return p.type == ServeType::kBf16 ? launch_type<Bf16>(p, stream) : launch_type<F16>(p, stream);
}

}  // namespace cp
