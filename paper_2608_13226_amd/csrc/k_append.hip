// Position rotation of queries and keys, and keys and values into a paged
// cache, in one pass.
//
// Pair i of a head (elements i and i + R/2, or 2i and 2i + 1) turns by
// position * inv_freq_i and grows by `magnitude`; elements from R on are
// copied.  Bound by memory: every element is read and written once.  A block
// works on one token, or on several that have few heads: a token's R/2 angles
// go to LDS once and serve all its heads.  6271 tokens of 32 + 32 heads of 64 in
// 31.7 us (4.85 TB/s), 1638 of 28 + 4 heads of 128 to e4m3 in 7.7 us.
//
// The angle is reduced to a fraction of a turn in float64 (32 bits of
// position and 24 of frequency do not fit a float32 product, whose error
// would reach whole hundredths of a radian at positions of 10^5), the sine
// and cosine of the fraction are float32.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// VEC consecutive elements of a head from element e on, into a query row or a
// cache row.  `den` is the head's scale (e4m3 caches).
template <class T, int VEC>
__device__ __forceinline__ void load_run(const void* p, int64_t i, float* x) {
  if constexpr (VEC == 8) load8<T>(p, i, x);
  else if constexpr (VEC == 4) load4<T>(p, i, x);
  else x[0] = load1<T>(p, i);
}
template <class C, int VEC>
__device__ __forceinline__ void store_run(void* p, int64_t i, float* x, float den) {
  if constexpr (sizeof(C) == 1) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] /= den;
  }
  if constexpr (VEC == 8) store8<C>(p, i, x);
  else if constexpr (VEC == 4) store4<C>(p, i, x);
  else store1<C>(p, i, x[0]);
}

// T: type of the projections, C: of the caches.  VEC = 8 needs 16-byte aligned
// rows, d % 8 == 0 and pairs that come in whole runs (rot % 16 == 0, or 8
// when interleaved); VEC = 4 half of each; VEC = 1 is for everything else.
// A block of 256 has `threads` for each of its tokens.
template <class T, class C, int VEC, bool INTER>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendParams p, int threads, int64_t first_block) {
  extern __shared__ float s_turns[];          // a token's [rot / 2] cosines, [rot / 2] sines
  const int tid = threadIdx.x % threads, mine = threadIdx.x / threads;
  const int64_t token = (first_block + blockIdx.x) * (256 / threads) + mine, t = min(token, p.tokens - 1);
  float* s_turn = s_turns + mine * p.rot;
  const int half = p.rot / 2;
  // All that is read before the angles is on its way together.  (The values
  // too, before the angles: 1638 tokens to e4m3 9.2 us instead of 8.3.)
  const double position = double(p.positions[t]);
  const int64_t slot = p.slots[t];
  const float frequency = tid < half ? p.inv_freq[tid] : 0.f;
  const bool here = token < p.tokens, keep = here && slot >= 0 && slot < p.pages * p.page;
  const int64_t pg = keep ? slot / p.page : 0;
  const int64_t off = keep ? slot - pg * p.page : 0;

  // A head's work: runs of pairs (two runs of VEC elements, or VEC = 1
  // interleaved pairs as two single ones), then runs of copied elements.
  const bool split = !INTER || VEC == 1;
  const int pair_runs = split ? half / VEC : p.rot / VEC;
  const int runs = pair_runs + (p.d - p.rot) / VEC;
  const int hq = p.q ? p.hq : 0;
  const int total = (hq + p.hk) * runs;
  const int first = blockIdx.y * threads + tid, step = gridDim.y * threads;
  for (int i = tid; i < half; i += threads) {
    double turns = position * (double(i == tid ? frequency : p.inv_freq[i]) * 0.15915494309189533576888);
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * float(turns), &s, &c);
    s_turn[i] = p.magnitude * c;
    s_turn[half + i] = p.magnitude * s;
  }
  __syncthreads();
  if (!here) return;
  for (int w = first; w < total; w += step) {
    const int head = w / runs, r = w - head * runs;
    const bool is_q = head < hq;
    const int kh = head - hq;
    if (!is_q && !keep) continue;
    const void* src = is_q ? p.q : p.k;
    const int64_t from = is_q ? t * p.q_stride + int64_t(head) * p.d : t * p.k_stride + int64_t(kh) * p.d;
    const int64_t to = is_q ? (t * p.hq + head) * p.d : ((pg * p.hk + kh) * p.page + off) * p.d;
    const float den = (!is_q && p.k_scale) ? p.k_scale[kh] : 1.f;
    auto put = [&](int e, float* x) {
      if (is_q) store_run<T, VEC>(p.q_out, to + e, x, 1.f);
      else store_run<C, VEC>(p.k_cache, to + e, x, den);
    };
    if (r >= pair_runs) {
      const int e = p.rot + (r - pair_runs) * VEC;
      float x[VEC];
      load_run<T, VEC>(src, from + e, x);
      put(e, x);
    } else if (split) {
      const int e1 = INTER ? 2 * r : r * VEC, e2 = INTER ? 2 * r + 1 : half + r * VEC;
      float a[VEC], b[VEC];
      load_run<T, VEC>(src, from + e1, a);
      load_run<T, VEC>(src, from + e2, b);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float c = s_turn[r * VEC + j], s = s_turn[half + r * VEC + j];
        const float x = a[j] * c - b[j] * s, y = b[j] * c + a[j] * s;
        a[j] = x;
        b[j] = y;
      }
      put(e1, a);
      put(e2, b);
    } else {
      const int e = r * VEC;
      float x[VEC];
      load_run<T, VEC>(src, from + e, x);
#pragma unroll
      for (int j = 0; j + 1 < VEC; j += 2) {
        const float c = s_turn[(e + j) / 2], s = s_turn[half + (e + j) / 2];
        const float a = x[j] * c - x[j + 1] * s, b = x[j + 1] * c + x[j] * s;
        x[j] = a;
        x[j + 1] = b;
      }
      put(e, x);
    }
  }
  if (!keep) return;
  const int vruns = p.d / VEC;
  // The values follow the rest, for the threads that have less of it.
  for (int w = (first - total % step + step) % step; w < p.hk * vruns; w += step) {
    const int kh = w / vruns, e = (w - kh * vruns) * VEC;
    float x[VEC];
    load_run<T, VEC>(p.v, t * p.v_stride + int64_t(kh) * p.d + e, x);
    store_run<C, VEC>(p.v_cache, ((pg * p.hk + kh) * p.page + off) * p.d + e, x, p.v_scale ? p.v_scale[kh] : 1.f);
  }
}

template <class T, class C, int VEC, bool INTER>
hipError_t launch(const KvAppendParams& p, hipStream_t stream) {
  // Few tokens: their heads are spread over more blocks, up to 2048, which find
  // the angles again, so that fewer threads have a second run to wait for (one
  // token of 64 + 16 heads of 128 4.9 -> 2.9 us, 300 tokens of them 5.9 -> 4.9;
  // with 4096 blocks 1638 tokens of 28 + 4 heads take 9.0 instead of 8.0).
  const int64_t work = (int64_t(p.q ? p.hq : 0) + 2 * p.hk) * (p.d / VEC);
  const unsigned y = unsigned(std::max<int64_t>(1, std::min<int64_t>(2048 / p.tokens, (work + 255) / 256)));
  // Many tokens of few heads: a block takes several, down to 256 blocks and as
  // long as a thread has at most four runs (19114 tokens of 2 + 2 heads of 64
  // 29.3 -> 10.2 us, 13119 of 4 + 4 of 96 22.9 -> 13.3, 2500 of 4 + 1 of 128 6.5 ->
  // 4.9; with up to eight runs 6271 of 32 + 32 of 64 35.8 instead of 34.5).
  int threads = 256;
  while (threads > 32 && threads / 2 >= work / 4 && p.tokens * (threads / 2) >= 256 * 256) threads /= 2;
  const int64_t per = 256 / threads;
  return launch_blocks((p.tokens + per - 1) / per, 256, [&](int64_t first, unsigned blocks) {
    kv_append_kernel<T, C, VEC, INTER><<<dim3(blocks, y), dim3(256), size_t(per) * p.rot * sizeof(float), stream>>>(p, threads, first);
  });
}

bool aligned(const void* q, int64_t stride, int bytes) {
  return reinterpret_cast<uintptr_t>(q) % bytes == 0 && stride * 2 % bytes == 0;
}

template <class T, class C, bool INTER>
hipError_t launch_width(const KvAppendParams& p, hipStream_t stream) {
  auto fits = [&](int vec) {
    return p.d % vec == 0 && p.rot % (INTER ? vec : 2 * vec) == 0 && (!p.q || aligned(p.q, p.q_stride, 2 * vec)) &&
           aligned(p.k, p.k_stride, 2 * vec) && aligned(p.v, p.v_stride, 2 * vec);
  };
  if (fits(8)) return launch<T, C, 8, INTER>(p, stream);
  return fits(4) ? launch<T, C, 4, INTER>(p, stream) : launch<T, C, 1, INTER>(p, stream);
}

template <class T, class C>
hipError_t launch_type(const KvAppendParams& p, hipStream_t stream) {
  return p.interleaved ? launch_width<T, C, true>(p, stream) : launch_width<T, C, false>(p, stream);
}

}  // namespace

hipError_t launch_kv_append(const KvAppendParams& p, hipStream_t stream) {
  if (p.type == ServeType::kBf16)
    return p.cache8 ? launch_type<Bf16, E4m3>(p, stream) : launch_type<Bf16, Bf16>(p, stream);
  return p.cache8 ? launch_type<F16, E4m3>(p, stream) : launch_type<F16, F16>(p, stream);
}

}  // namespace cp
