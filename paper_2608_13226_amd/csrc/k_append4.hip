// Position rotation of queries and keys, and keys and values into a paged cache
// of 4 bits, in one pass.
//
// A block of 32 elements x is held as s = 2^e, the smallest power (of those
// whose values are normal and finite in T) with max |x| <= 6 s, and the codes
// of x / s rounded to nearest, ties to the even code; what lies beyond 6 s of the
// largest power becomes that.  Every element is read once and written once, queries in
// 16 bits, keys and values in 4.25; what bounds it are the vector instructions (6271
// tokens of 32 + 2 x 32 heads of 64 in 27.7 us, 4.2 TB/s; they issue in 61 % of the cycles of busy compute units).
//
// Codes are those of the key rotated in float64: a float32 rotation would put
// one code in 10^6 on the other side of a border (as a magnitude of 1.2 rounded to
// float32 did with whole blocks at position 0, whose largest is 6 times a power).  The angle, position *
// inv_freq, is reduced to a fraction of a turn with 1 / 2 pi in two parts, so that
// it is off by the rounding of the product alone.  A key goes to float32 rounded to
// odd (towards zero, last bit set where something was cut), which keeps it on
// its side of every border.  Queries are rotated in float32, as in kv_append.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// float64 to float32, rounded to odd at 21 bits after the leading one: of the 31 that go, whether any
// was set stays in the last one of the others, and the conversion is exact down to 2^-128, below all borders (the
// lowest is 2^-127, where float32 has 22 such bits).  (Past float32's range: infinite.)
__device__ __forceinline__ float round_odd(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return float(__builtin_bit_cast(double, (b & 0xffffffff00000000u) | (uint32_t(b) ? 0x80000000u : 0u)));
}

// Eight elements from element i on, as they are stored.
template <bool WHOLE>
__device__ __forceinline__ u32x4 load_run(const uint16_t* p) {
  if constexpr (WHOLE) return *reinterpret_cast<const u32x4*>(p);
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = uint32_t(p[2 * j]) | uint32_t(p[2 * j + 1]) << 16;
  return w;
}
template <class T>
__device__ __forceinline__ void widen8(u32x4 w, float* x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = unpack2<T>(w[j]);
    x[2 * j] = f.x;
    x[2 * j + 1] = f.y;
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

// Elements e + 0..7 of a head, which lie at `run`, turned where they are below rot; `own` holds
// them, cosines and sines are the pairs'.  R: float or double.
template <class T, bool INTER, bool WHOLE, class R>
__device__ __forceinline__ void turn_run(const uint16_t* run, int e, int rot, const R* cosines, const R* sines, const float* own, R* y) {
  const int half = rot / 2;
  if constexpr (WHOLE && INTER) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const R c = cosines[e / 2 + j / 2], s = sines[e / 2 + j / 2], a = own[j], b = own[j + 1];
      y[j] = a * c - b * s;
      y[j + 1] = b * c + a * s;
    }
  } else if constexpr (WHOLE) {
    const bool second = e >= half;
    const int i0 = second ? e - half : e;
    float other[8];
    widen8<T>(load_run<true>(run + (second ? -half : half)), other);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const R c = cosines[i0 + j], s = second ? -sines[i0 + j] : sines[i0 + j];
      y[j] = R(own[j]) * c - R(other[j]) * s;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = e + j;
      y[j] = own[j];
      if (i < rot) {
        const bool second = INTER ? i % 2 != 0 : i >= half;
        const int pair = INTER ? i / 2 : second ? i - half : i, to = INTER ? (second ? -1 : 1) : second ? -half : half;
        const R c = cosines[pair], s = second ? -sines[pair] : sines[pair], other = load1<T>(run, j + to);
        y[j] = R(own[j]) * c - other * s;
      }
    }
  }
}

// A block of 256 has 2^shift threads, whole waves, for each of its tokens.  A thread has runs of
// eight elements, queries', then keys', then values' (a wave's are of one tensor but for two, which takes
// a third of the index arithmetic of runs in one sequence); the first of each are on their way while
// the block finds the token's angles.  WHOLE: rows are 16-byte aligned and no run holds the
// end of a head's turned part or of its half.
template <class T, bool INTER, bool WHOLE>
__global__ __launch_bounds__(256) void kv_append4_kernel(KvAppend4Params p, int shift, int64_t first_block) {
  extern __shared__ double s_turns[];         // a token's [rot / 2] cosines, sines, and both again as floats
  const int threads = 1 << shift, tid = int(threadIdx.x) & (threads - 1);
  const int mine = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> shift);
  const int64_t token = (first_block + blockIdx.x) * (256 >> shift) + mine, t = min(token, p.tokens - 1);
  const int half = p.rot / 2;
  double *s_cos = s_turns + int64_t(mine) * half * 3, *s_sin = s_cos + half;
  float *s_cosf = reinterpret_cast<float*>(s_sin + half), *s_sinf = s_cosf + half;
  const double position = double(p.positions[t]);
  const int64_t slot = p.slots[t];

  const int runs = p.d / 8, q_runs = p.q ? p.hq * runs : 0, k_runs = p.hk * runs;
  const int step = int(gridDim.y) * threads, at = int(blockIdx.y) * threads + tid;
  // The thread's first run of a tensor before which the threads have had `before`.
  auto first_of = [&](int before) {
    const int w = at - before % step;
    return w < 0 ? w + step : w;
  };
  const int q0 = at, k0 = first_of(q_runs), v0 = first_of(q_runs + k_runs);
  const uint16_t* q = static_cast<const uint16_t*>(p.q) + t * p.q_stride;
  const uint16_t* k = static_cast<const uint16_t*>(p.k) + t * p.k_stride;
  const uint16_t* v = static_cast<const uint16_t*>(p.v) + t * p.v_stride;
  u32x4 raw_q = {0, 0, 0, 0}, raw_k = raw_q, raw_v = raw_q;
  if (q0 < q_runs) raw_q = load_run<WHOLE>(q + q0 * 8);
  if (k0 < k_runs) raw_k = load_run<WHOLE>(k + k0 * 8);
  if (v0 < k_runs) raw_v = load_run<WHOLE>(v + v0 * 8);

  for (int i = tid; i < half; i += threads) {
    const double angle = position * double(p.inv_freq[i]);
    // angle / 2 pi less its whole turns; 1 / 2 pi = high + low.
    const double high = 0.15915494309189535, low = -9.839338337591243e-18;
    const double turns = angle * high, rest = fma(angle, high, -turns) + angle * low;
    double s, c;
    sincospi(2.0 * ((turns - rint(turns)) + rest), &s, &c);
    c *= p.magnitude;
    s *= p.magnitude;
    s_cos[i] = c;
    s_sin[i] = s;
    s_cosf[i] = float(c);
    s_sinf[i] = float(s);
  }
  lds_sync();
  if (token >= p.tokens) return;

  uint16_t* q_out = static_cast<uint16_t*>(p.q_out) + t * (p.hq * int64_t(p.d));
  for (int w = q0; w < q_runs; w += step) {
    const int e = (w - int(p.by_runs(unsigned(w))) * runs) * 8;
    if (w != q0) raw_q = load_run<WHOLE>(q + w * 8);
    if (e < p.rot) {
      float x[8], y[8];
      widen8<T>(raw_q, x);
      turn_run<T, INTER, WHOLE, float>(q + w * 8, e, p.rot, s_cosf, s_sinf, x, y);
#pragma unroll
      for (int j = 0; j < 4; ++j) raw_q[j] = pack2<T>(y[2 * j], y[2 * j + 1]);
    }
    *reinterpret_cast<u32x4*>(q_out + w * 8) = raw_q;
  }
  if (slot < 0 || slot >= p.pages * p.page) return;
  const int64_t pg = page_of(slot, p.page, p.by_page), row0 = pg * p.hk * p.page + (slot - pg * p.page);
  // Run w of keys or values as a block's part.
  auto put = [&](int w, const float* x, uint8_t* cache, uint8_t* scale) {
    const int head = int(p.by_runs(unsigned(w))), e = (w - head * runs) * 8;
    uint32_t exponent;
    const uint32_t codes = cut_block<T>(x, &exponent);
    const int64_t row = row0 + int64_t(head) * p.page;
    *reinterpret_cast<uint32_t*>(cache + row * (p.d / 2) + e / 2) = codes;
    if (e % kBlock4 == 0) scale[row * (p.d / kBlock4) + e / kBlock4] = uint8_t(exponent);
  };
  for (int w = k0; w < k_runs; w += step) {
    const int e = (w - int(p.by_runs(unsigned(w))) * runs) * 8;
    if (w != k0) raw_k = load_run<WHOLE>(k + w * 8);
    float x[8];
    widen8<T>(raw_k, x);
    if (e < p.rot) {
      double y[8];
      turn_run<T, INTER, WHOLE, double>(k + w * 8, e, p.rot, s_cos, s_sin, x, y);
      float most = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = round_odd(y[j]);
        most = fmaxf(most, fabsf(x[j]));
      }
      if (most > 3e38f) {
        // What is finite but past float32's range counts as its largest number.
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (fabs(y[j]) < __builtin_inf()) x[j] = round_odd(fmin(fmax(y[j], -3.4028234663852886e38), 3.4028234663852886e38));
      }
    }
    put(w, x, p.k_cache, p.k_scale);
  }
  for (int w = v0; w < k_runs; w += step) {
    if (w != v0) raw_v = load_run<WHOLE>(v + w * 8);
    float x[8];
    widen8<T>(raw_v, x);
    put(w, x, p.v_cache, p.v_scale);
  }
}

template <class T, bool INTER, bool WHOLE>
hipError_t launch(const KvAppend4Params& p, hipStream_t stream) {
  // As kv_append: few tokens are spread over more blocks, many tokens of few heads share one.
  const int64_t work = (int64_t(p.q ? p.hq : 0) + 2 * p.hk) * (p.d / 8);
  const unsigned y = unsigned(std::max<int64_t>(1, std::min<int64_t>(2048 / p.tokens, (work + 255) / 256)));
  int shift = 8;
  while (shift > 6 && (1 << shift) / 2 >= work / 4 && p.tokens * (1 << shift) / 2 >= 256 * 256) --shift;
  const int64_t per = 256 >> shift;
  return launch_blocks((p.tokens + per - 1) / per, 256, [&](int64_t first, unsigned blocks) {
    kv_append4_kernel<T, INTER, WHOLE><<<dim3(blocks, y), dim3(256), size_t(per) * p.rot * 12, stream>>>(p, shift, first);
  });
}

bool aligned(const void* q, int64_t stride) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && stride % 8 == 0; }

template <class T>
hipError_t launch_type(const KvAppend4Params& p, hipStream_t stream) {
  const bool whole = (!p.q || aligned(p.q, p.q_stride)) && aligned(p.k, p.k_stride) && aligned(p.v, p.v_stride) &&
                     p.rot % (p.interleaved ? 8 : 16) == 0;
  if (p.interleaved) return whole ? launch<T, true, true>(p, stream) : launch<T, true, false>(p, stream);
  return whole ? launch<T, false, true>(p, stream) : launch<T, false, false>(p, stream);
}

}  // namespace

hipError_t launch_kv_append4(const KvAppend4Params& p, hipStream_t stream) {
  return p.type == ServeType::kBf16 ? launch_type<Bf16>(p, stream) : launch_type<F16>(p, stream);
}

}  // namespace cp
