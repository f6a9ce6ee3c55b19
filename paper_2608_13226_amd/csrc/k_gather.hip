// Keys and values of given slots of a paged cache as dense rows: the cache's
// append undone.  Bound by memory; a thread has runs of eight elements of a
// key or value, 16 bits of which are copied, 8 bits widened and scaled in
// float32, 4 bits widened with their block's power.  65537 tokens of 8 heads of
// 128 from e4m3 in 79 us (5.1 TB/s; 107 with one run a thread), 65536 of 4 heads from
// 4 bits in 40 (4.2 TB/s) from memory, 27 where the codes are still in the caches; divisions
// took a tenth more.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// VEC = 8 needs d % 8 == 0; VEC = 1 is for the rest.  A token's 2 hk heads have runs =
// d / VEC each; a thread takes kAhead runs, 256 apart, so that its loads are under way together.
constexpr int kAhead = 4;

template <class T, int BITS, int VEC>
struct Run {
  static constexpr int kWords = VEC == 1 ? 1 : BITS / 4;
  uint32_t w[kWords];
  float scale;

  __device__ __forceinline__ void load(const KvGatherParams& p, bool is_v, int64_t row, int kh, int e) {
    const uint8_t* cache = static_cast<const uint8_t*>(is_v ? p.v_cache : p.k_cache);
    const void* scales = is_v ? p.v_scale : p.k_scale;
    if constexpr (BITS == 16) {
      const uint16_t* x = reinterpret_cast<const uint16_t*>(cache) + row * p.d + e;
      if constexpr (VEC == 1) {
        w[0] = *x;
      } else {
        const u32x4 v = *reinterpret_cast<const u32x4*>(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v[i];
      }
    } else if constexpr (BITS == 8) {
      const uint8_t* x = cache + row * p.d + e;
      if constexpr (VEC == 1) {
        w[0] = *x;
      } else {
        const u32x2 v = *reinterpret_cast<const u32x2*>(x);
        w[0] = v[0];
        w[1] = v[1];
      }
      scale = scales ? static_cast<const float*>(scales)[kh] : 1.f;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(cache + row * (p.d / 2) + e / 2);
      scale = power_of(static_cast<const uint8_t*>(scales)[row * (p.d / kBlock4) + e / kBlock4]);
    }
  }
  __device__ __forceinline__ void store(void* out, int64_t to) const {
    if constexpr (VEC == 1) {
      if constexpr (BITS == 16) static_cast<uint16_t*>(out)[to] = uint16_t(w[0]);
      else store1<T>(out, to, unpack2<Bf16>(widen2<Bf16, false>(w[0])).x * scale);
    } else if constexpr (BITS == 16) {
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + to) = u32x4{w[0], w[1], w[2], w[3]};
    } else if constexpr (BITS == 8) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 lo = unpack2<Bf16>(widen2<Bf16, false>(w[i])), hi = unpack2<Bf16>(widen2<Bf16, true>(w[i]));
        x[4 * i] = lo.x * scale;
        x[4 * i + 1] = lo.y * scale;
        x[4 * i + 2] = hi.x * scale;
        x[4 * i + 3] = hi.y * scale;
      }
      store8<T>(out, to, x);
    } else {
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + to) =
          u32x4{open2<T>(w[0], scale, 0), open2<T>(w[0], scale, 1), open2<T>(w[0], scale, 2), open2<T>(w[0], scale, 3)};
    }
  }
};

// `tokens` tokens a block, of a_token runs each.
template <class T, int BITS, int VEC>
__global__ __launch_bounds__(256) void kv_gather_kernel(KvGatherParams p, Divide by_token, Divide by_runs, int tokens, int64_t first_block) {
  const unsigned runs = unsigned(p.d / VEC), half = unsigned(p.hk) * runs, a_token = 2 * half;
  const int64_t t0 = (first_block + blockIdx.x) * tokens;
  const unsigned total = unsigned(min(int64_t(tokens), p.tokens - t0)) * a_token;
  for (unsigned w0 = threadIdx.x; w0 < total; w0 += 256 * kAhead) {
    Run<T, BITS, VEC> x[kAhead];
    int64_t slot[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) slot[i] = p.slots[t0 + by_token(min(w0 + i * 256, total - 1))];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const unsigned w = min(w0 + i * 256, total - 1), r = w - by_token(w) * a_token, in = r < half ? r : r - half;
      const unsigned kh = by_runs(in), e = (in - kh * runs) * VEC;
      const int64_t at = slot[i] >= 0 && slot[i] < p.pages * p.page ? slot[i] : 0;
      const int64_t pg = page_of(at, p.page, p.by_page);
      x[i].load(p, r >= half, (pg * p.hk + kh) * p.page + (at - pg * p.page), int(kh), int(e));
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const unsigned w = w0 + i * 256;
      if (w >= total) break;
      const unsigned token = by_token(w), r = w - token * a_token, in = r < half ? r : r - half;
      if (slot[i] < 0 || slot[i] >= p.pages * p.page) x[i] = {};
      x[i].store(r < half ? p.k_out : p.v_out, (t0 + token) * half * VEC + in * VEC);
    }
  }
}

template <class T, int BITS, int VEC>
hipError_t launch(const KvGatherParams& p, hipStream_t stream) {
  // Up to 1024 runs a block, a token's at least.
  const int64_t a_token = 2 * int64_t(p.hk) * (p.d / VEC);
  const int tokens = int(std::max<int64_t>(1, 256 * kAhead / a_token));
  return launch_blocks((p.tokens + tokens - 1) / tokens, 256, [&](int64_t first, unsigned blocks) {
    kv_gather_kernel<T, BITS, VEC><<<dim3(blocks), dim3(256), 0, stream>>>(p, Divide(a_token), Divide(p.d / VEC), tokens, first);
  });
}

template <class T>
hipError_t launch_type(const KvGatherParams& p, hipStream_t stream) {
  if (p.held == ServeType::kE2m1) return launch<T, 4, 8>(p, stream);
  if (p.held == ServeType::kE4m3) return p.d % 8 == 0 ? launch<T, 8, 8>(p, stream) : launch<T, 8, 1>(p, stream);
  return p.d % 8 == 0 ? launch<T, 16, 8>(p, stream) : launch<T, 16, 1>(p, stream);
}

}  // namespace

hipError_t launch_kv_gather(const KvGatherParams& p, hipStream_t stream) {
  return p.type == ServeType::kBf16 ? launch_type<Bf16>(p, stream) : launch_type<F16>(p, stream);
}

}  // namespace cp
