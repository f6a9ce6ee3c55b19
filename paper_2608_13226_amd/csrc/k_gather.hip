// Keys and values of given slots of a paged cache as dense rows: the cache's
// append undone.  Bound by memory; a thread has runs of eight elements of a
// key or value, 16 bits of which are copied, 8 bits widened and scaled in
// float32, 4 bits widened with their block's power.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

// VEC = 8 needs d % 8 == 0; VEC = 1 is for the rest.  A token's 2 hk heads have runs = d / VEC each.
template <class T, int BITS, int VEC>
__global__ __launch_bounds__(256) void kv_gather_kernel(KvGatherParams p, int64_t first_block) {
  const int64_t runs = p.d / VEC, a_token = 2 * int64_t(p.hk) * runs;
  const int64_t w = (first_block + blockIdx.x) * 256 + threadIdx.x;
  const int64_t token = w / a_token;
  if (token >= p.tokens) return;
  int64_t r = w - token * a_token;
  const bool is_v = r >= int64_t(p.hk) * runs;
  if (is_v) r -= int64_t(p.hk) * runs;
  const int kh = int(r / runs), e = int(r - kh * runs) * VEC;
  const int64_t slot = p.slots[token], to = (token * p.hk + kh) * p.d + e;
  void* out = is_v ? p.v_out : p.k_out;
  if (slot < 0 || slot >= p.pages * p.page) {
    if constexpr (VEC == 8) *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + to) = u32x4{0, 0, 0, 0};
    else static_cast<uint16_t*>(out)[to] = 0;
    return;
  }
  const int64_t pg = slot / p.page, row = (pg * p.hk + kh) * p.page + (slot - pg * p.page);
  const uint8_t* cache = static_cast<const uint8_t*>(is_v ? p.v_cache : p.k_cache);
  if constexpr (BITS == 16) {
    if constexpr (VEC == 8)
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + to) = *reinterpret_cast<const u32x4*>(cache + (row * p.d + e) * 2);
    else static_cast<uint16_t*>(out)[to] = reinterpret_cast<const uint16_t*>(cache)[row * p.d + e];
  } else if constexpr (BITS == 8) {
    const float* scales = static_cast<const float*>(is_v ? p.v_scale : p.k_scale);
    const float scale = scales ? scales[kh] : 1.f;
    if constexpr (VEC == 8) {
      const u32x2 v = *reinterpret_cast<const u32x2*>(cache + row * p.d + e);
      float x[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 lo = unpack2<Bf16>(widen2<Bf16, false>(v[i])), hi = unpack2<Bf16>(widen2<Bf16, true>(v[i]));
        x[4 * i] = lo.x * scale;
        x[4 * i + 1] = lo.y * scale;
        x[4 * i + 2] = hi.x * scale;
        x[4 * i + 3] = hi.y * scale;
      }
      store8<T>(out, to, x);
    } else {
      store1<T>(out, to, unpack2<Bf16>(widen2<Bf16, false>(cache[row * p.d + e])).x * scale);
    }
  } else {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(cache + row * (p.d / 2) + e / 2);
    const uint8_t* exps = static_cast<const uint8_t*>(is_v ? p.v_scale : p.k_scale);
    const float s = power_of(exps[row * (p.d / kBlock4) + e / kBlock4]);
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + to) = u32x4{open2<T>(v, s, 0), open2<T>(v, s, 1), open2<T>(v, s, 2), open2<T>(v, s, 3)};
  }
}

template <class T, int BITS, int VEC>
hipError_t launch(const KvGatherParams& p, hipStream_t stream) {
  const int64_t work = p.tokens * 2 * p.hk * (p.d / VEC);
  return launch_blocks((work + 255) / 256, 256, [&](int64_t first, unsigned blocks) {
    kv_gather_kernel<T, BITS, VEC><<<dim3(blocks), dim3(256), 0, stream>>>(p, first);
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
