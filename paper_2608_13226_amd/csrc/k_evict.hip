// Eviction from a paged cache: of each sequence and key-value head the tokens of
// largest mass stay, and close the gaps that the others leave.
//
// With n tokens of which m = keep stay (n > keep), the first `sink` and the last
// `recent` among them, f = m - recent.  Tokens below f that stay do not move; those
// from f to n - recent move to the places below f that fall vacant, in order; the
// last `recent` go to f and on, in order.  So the rows that move are at most as
// many as those that leave, and the last ones, and not the whole cache.
//
//   select  a block a (sequence, head): the mass of rank m - sink - recent by its
//           bits, eight at a time; then, in order of the tokens, who leaves, who
//           moves and the new order.
//   move    rows to vacant places, and the new masses.  All come from f on and
//           go below f, so no row is read after it was written.
//   shift   the last rows, once the places at f are empty; in ascending runs, each
//           read whole before it is written, since they may overlap.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

constexpr int kSelect = 1024;

// Where the workspace holds what, for each (sequence, head), in 32-bit words.
struct Lists {
  int64_t places;                 // most places that can fall vacant
  int64_t vacant, movers, count, mass, stride;
};
__host__ __device__ inline Lists lists_of(int64_t keep, int64_t recent, int64_t max_length) {
  Lists l;
  const int64_t a = keep - recent, b = max_length - keep;
  l.places = a < b ? a : b;
  if (l.places < 0) l.places = 0;
  l.count = 0;
  l.vacant = 1;
  l.movers = l.vacant + l.places;
  l.mass = l.movers + l.places;
  l.stride = l.mass + (keep < max_length ? keep : max_length);
  return l;
}

// A mass as a number in the order of masses: NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t rank_of(float m) {
  if (m != m) return 0u;
  const uint32_t b = __float_as_uint(m + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum of one number a thread over the block's lower threads, and over all.
__device__ __forceinline__ int block_scan(int x, int* s_part, int* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int sum = x;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == kWave - 1) s_part[wave] = sum;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kSelect / kWave; ++i) {
    const int v = s_part[i];
    if (i < wave) before += v;
    all += v;
  }
  __syncthreads();
  *total = all;
  return before + sum - x;
}

__device__ __forceinline__ int tokens_of(const KvEvictParams& p, int b) { return max(0, int(min(int64_t(p.lengths[b]), p.max_length))); }

__global__ __launch_bounds__(kSelect) void evict_select_kernel(KvEvictParams p) {
  __shared__ int s_hist[256];
  __shared__ int s_part[kSelect / kWave];
  __shared__ uint32_t s_digit, s_left;
  const int kh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int n = tokens_of(p, b), keep = int(p.keep), recent = int(p.recent), sink = int(p.sink);
  const int64_t head = int64_t(b) * p.hk + kh;
  const Lists l = lists_of(p.keep, p.recent, p.max_length);
  uint32_t* ws = static_cast<uint32_t*>(p.workspace) + head * l.stride;
  int *vacant = reinterpret_cast<int*>(ws + l.vacant), *movers = reinterpret_cast<int*>(ws + l.movers);
  float* fresh = reinterpret_cast<float*>(ws + l.mass);
  const float* mass = p.mass + head * p.span;
  int32_t* kept = p.kept + head * p.keep;
  if (n <= keep) {
    for (int64_t j = tid; j < keep; j += kSelect) {
      kept[j] = j < n ? int(j) : -1;
      if (j < n) fresh[j] = mass[j];
    }
    if (tid == 0) ws[l.count] = 0u;
    return;
  }
  // Of the tokens in [sink, end) `want` stay: those whose rank is above `border`, and
  // the first `ties` of those at it.
  const int end = n - recent, want = keep - recent - sink, front = keep - recent;
  uint32_t border = 0u;
  int ties = 0;
  if (want > 0) {
    uint32_t left = uint32_t(want);
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelect) s_hist[i] = 0;
      __syncthreads();
      for (int j = sink + tid; j < end; j += kSelect) {
        const uint32_t r = rank_of(mass[j]);
        if (shift == 24 || r >> (shift + 8) == border >> (shift + 8)) atomicAdd(&s_hist[r >> shift & 255u], 1);
      }
      __syncthreads();
      // The digit at which the counts from the highest on reach what is left.
      if (tid < kWave) {
        int c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += c[i] = s_hist[255 - (tid * 4 + i)];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
          const int y = __shfl_up(upto, o);
          if (tid >= o) upto += y;
        }
        int before = upto - sum;
        if (before < int(left) && int(left) <= upto) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (before < int(left) && int(left) <= before + c[i]) {
              s_digit = 255 - (tid * 4 + i);
              s_left = left - before;
            }
            before += c[i];
          }
        }
      }
      __syncthreads();
      border |= s_digit << shift;
      left = s_left;
      __syncthreads();
    }
    ties = int(left);
  }
  // In order: counts of ties, vacant places and movers up to each token.
  int seen = 0, gaps = 0, moved = 0;
  for (int j0 = 0; j0 < end; j0 += kSelect) {
    const int j = j0 + tid;
    const bool here = j < end;
    const float m = here ? mass[j] : 0.f;
    const uint32_t r = rank_of(m);
    const bool inner = here && j >= sink;
    const bool tie = inner && want > 0 && r == border;
    int total;
    const int rank = seen + block_scan(tie, s_part, &total);
    seen += total;
    const bool stays = here && (j < sink || (want > 0 && (r > border || (tie && rank < ties))));
    const bool gap = here && !stays && j < front, goes = stays && j >= front;
    // Both counts in one number: below the front only gaps, from it on only movers,
    // but for the run in which it lies.
    int both;
    const int at = block_scan(gap | int(goes) << 16, s_part, &both);
    if (gap) vacant[gaps + (at & 0xffff)] = j;
    if (goes) movers[moved + (at >> 16)] = j;
    gaps += both & 0xffff;
    moved += both >> 16;
    if (stays && j < front) {
      kept[j] = j;
      fresh[j] = m;
    }
  }
  __syncthreads();
  for (int i = tid; i < gaps; i += kSelect) {
    const int from = movers[i], to = vacant[i];
    kept[to] = from;
    fresh[to] = mass[from];
  }
  for (int i = tid; i < recent; i += kSelect) {
    kept[front + i] = end + i;
    fresh[front + i] = mass[end + i];
  }
  if (tid == 0) ws[l.count] = uint32_t(gaps);
}

// One row of codes, values or exponents from one place to another, `units` of U, one of them.
struct Place {
  const KvEvictParams& p;
  int b, kh;
  // Row of token t.
  __device__ __forceinline__ int64_t row(int t) const {
    const int page = t / p.page;
    const unsigned entry = min(unsigned(p.table[int64_t(b) * p.width + page]), unsigned(p.pages - 1));
    return (int64_t(entry) * p.hk + kh) * p.page + (t - page * p.page);
  }
};

// The rows' copies: `lanes` threads a pair of places.
constexpr int kMoveRows = 32;
template <class U>
__device__ __forceinline__ void copy_row(void* base, int64_t to, int64_t from, int units, int lane, int lanes) {
  U* x = static_cast<U*>(base);
  for (int i = lane; i < units; i += lanes) x[to * units + i] = x[from * units + i];
}

template <class U>
__global__ __launch_bounds__(256) void evict_move_kernel(KvEvictParams p) {
  const int kh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int64_t head = int64_t(b) * p.hk + kh;
  const Lists l = lists_of(p.keep, p.recent, p.max_length);
  const uint32_t* ws = static_cast<const uint32_t*>(p.workspace) + head * l.stride;
  const int count = int(ws[l.count]);
  const int *vacant = reinterpret_cast<const int*>(ws + l.vacant), *movers = reinterpret_cast<const int*>(ws + l.movers);
  const float* fresh = reinterpret_cast<const float*>(ws + l.mass);
  const int n = tokens_of(p, b), m = min(int64_t(n), p.keep);
  float* mass = p.mass_out + head * p.span;
  for (int64_t j = int64_t(blockIdx.x) * 256 + tid; j < p.span; j += int64_t(gridDim.x) * 256) mass[j] = j < m ? fresh[j] : 0.f;
  if (kh == 0 && blockIdx.x == 0 && tid == 0) p.lengths_out[b] = m;
  const Place place = {p, b, kh};
  const int units = p.row_bytes / int(sizeof(U));
  const int lane = tid % 8, group = tid / 8;
  for (int i = blockIdx.x * kMoveRows + group; i < count; i += int(gridDim.x) * kMoveRows) {
    const int64_t to = place.row(vacant[i]), from = place.row(movers[i]);
    copy_row<U>(p.k_cache, to, from, units, lane, 8);
    copy_row<U>(p.v_cache, to, from, units, lane, 8);
    if (p.exp_bytes) {
      copy_row<uint8_t>(p.k_exps, to, from, p.exp_bytes, lane, 8);
      copy_row<uint8_t>(p.v_exps, to, from, p.exp_bytes, lane, 8);
    }
  }
}

template <class U>
__global__ __launch_bounds__(256) void evict_shift_kernel(KvEvictParams p) {
  const int kh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int n = tokens_of(p, b), keep = int(p.keep), recent = int(p.recent);
  if (n <= keep) return;
  const Place place = {p, b, kh};
  // Block x has the keys, the values, or the exponents of either.
  void* base = blockIdx.x == 0 ? p.k_cache : blockIdx.x == 1 ? p.v_cache : blockIdx.x == 2 ? static_cast<void*>(p.k_exps) : static_cast<void*>(p.v_exps);
  const int units = blockIdx.x < 2 ? p.row_bytes / int(sizeof(U)) : p.exp_bytes;
  // Units in the order of rows: a run of 256 is read before any of it is written, and
  // a later run's rows lie behind all rows written so far.
  const int64_t total = int64_t(recent) * units;
  for (int64_t i0 = 0; i0 < total; i0 += 256) {
    const int64_t i = i0 + tid;
    const bool here = i < total;
    const int r = here ? int(i / units) : 0, u = here ? int(i - int64_t(r) * units) : 0;
    const int64_t from = place.row(n - recent + r) * units + u, to = place.row(keep - recent + r) * units + u;
    U x;
    uint8_t e = 0;
    if (here) {
      if (blockIdx.x < 2) x = static_cast<const U*>(base)[from];
      else e = static_cast<const uint8_t*>(base)[from];
    }
    __syncthreads();
    if (here) {
      if (blockIdx.x < 2) static_cast<U*>(base)[to] = x;
      else static_cast<uint8_t*>(base)[to] = e;
    }
    __syncthreads();
  }
}

template <class U>
hipError_t launch(const KvEvictParams& p, hipStream_t stream) {
  const Lists l = lists_of(p.keep, p.recent, p.max_length);
  evict_select_kernel<<<dim3(unsigned(p.hk), unsigned(p.batch)), dim3(kSelect), 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t want = std::max((l.places + kMoveRows - 1) / kMoveRows, (p.span + 2047) / 2048);
  const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(want, 4096 / (int64_t(p.hk) * p.batch)));
  evict_move_kernel<U><<<dim3(unsigned(blocks), unsigned(p.hk), unsigned(p.batch)), dim3(256), 0, stream>>>(p);
  e = hipGetLastError();
  if (e != hipSuccess || p.recent == 0 || p.max_length <= p.keep) return e;
  evict_shift_kernel<U><<<dim3(p.exp_bytes ? 4 : 2, unsigned(p.hk), unsigned(p.batch)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t evict_workspace_bytes(int64_t batch, int64_t hk, int64_t keep, int64_t recent, int64_t max_length) {
  return size_t(batch * hk * lists_of(keep, recent, max_length).stride) * sizeof(uint32_t);
}

hipError_t launch_kv_evict(const KvEvictParams& p, hipStream_t stream) {
  if (p.row_bytes % 16 == 0) return launch<u32x4>(p, stream);
  return launch<u32x2>(p, stream);
}

}  // namespace cp
