// Eviction from a paged cache: of each sequence and key-value head the tokens of
// largest mass stay, and close the gaps that the others leave.
//
// With n tokens of which keep stay (n > keep), the first `sink` and the last
// `recent` among them, front = keep - recent.  Tokens below the front that stay do not
// move; those from it to n - recent move to the places below it that fall vacant, in
// order; the last `recent` go to the front and on, in order.  So the rows that move are
// at most as many as those that leave, and the last ones, and not the whole cache.
//
// Who stays: of the tokens in [sink, n - recent) the want = front - sink of largest
// rank (a mass as a whole number in the order of masses), found digit by digit from
// counts of them; of those at the last rank the earlier.  The order of tokens comes
// from counts as well, so nothing depends on the order of atomics.
//
//   evict_one    up to 16384 tokens: a block a (sequence, head) selects, the ranks in LDS;
//                where few rows move, it moves them too, and one launch does it all
//   longer sequences have their tokens in up to 64 chunks:
//   evict_count  a chunk's counts of the rank's highest 10 bits
//   evict_bucket the value of those at which the rank wanted lies; a chunk's tokens that
//                have it, its counts of those above
//   evict_border the rank itself, from the tokens with that value, by every block for
//                itself; then its chunk's vacant places and movers
//   evict_move   rows and masses to vacant places.  All come from the front on and go
//                below it, so no row is read after it was written.
//   evict_shift  the last rows, once the places at the front are empty
//
// Bound by the launches and barriers between dependent steps: 8 sequences of up to 1702
// tokens of 4 heads, 64 of each out, 11.4 us; 131072 tokens of 4 heads halved 50 us
// without the gaps between five launches, of which the rows, in scattered pieces of 64
// and 4 bytes, take 19.
#include <algorithm>

#include "launch.h"
#include "serve.h"

namespace cp {
namespace {

constexpr int kSelect = 1024, kWaves = kSelect / kWave;

// A mass as a number in the order of masses: NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t rank_of(float m) {
  if (m != m) return 0u;
  const uint32_t b = __float_as_uint(m + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ int tokens_of(const KvEvictParams& p, int b) { return max(0, int(min(int64_t(p.lengths[b]), p.max_length))); }

// How many lanes below this one have their bit in `ballot`.
__device__ __forceinline__ int lanes_below(unsigned long long ballot) {
  return int(__builtin_amdgcn_mbcnt_hi(unsigned(ballot >> 32), __builtin_amdgcn_mbcnt_lo(unsigned(ballot), 0u)));
}

// Sum over this lane and the lower ones; every lane of the wave is active.
__device__ __forceinline__ int wave_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // from 1, 2, 4 and 8 lanes below in a row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // lane 15 of a row to the next, rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // lane 31 to rows 2 and 3
  return x;
}

// Of one number a wave of the block: the sum of the lower waves', and of all.  A lane takes a
// wave's: all sixteen in each lane took a third of a selection's time.
__device__ __forceinline__ int waves_below(const int* part, int wave, int* all = nullptr) {
  static_assert(kWaves == 16, "a row of lanes has the waves");
  const int v = part[threadIdx.x % kWaves];
  int upto = v;
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, false);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, false);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, false);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, false);
  if (all) *all = __builtin_amdgcn_readlane(upto, kWaves - 1);
  return __builtin_amdgcn_readlane(upto, wave) - __builtin_amdgcn_readlane(v, wave);
}

// Counts of a digit with BINS values, COPIES each.
template <int BINS, int COPIES>
struct Digits {
  static constexpr int kPer = BINS / kSelect;
  int count[BINS * COPIES], upto[kWaves], left;
  uint32_t digit;

  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < BINS * COPIES; i += kSelect) count[i] = 0;
  }
  __device__ __forceinline__ void add(uint32_t d) { atomicAdd(&count[d * COPIES + threadIdx.x % COPIES], 1); }

  // The digit at which the counts from the highest on reach `rest` (1 <= rest <= their
  // sum), and how many are left at it.  The block has synchronised after its last add.
  __device__ __forceinline__ uint32_t find(int& rest) {
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave), top = BINS - 1 - int(threadIdx.x) * kPer;
    int c[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      c[i] = 0;
#pragma unroll
      for (int e = 0; e < COPIES; ++e) c[i] += count[(top - i) * COPIES + e];
      sum += c[i];
    }
    const int here = wave_upto(sum);
    if (threadIdx.x % kWave == kWave - 1) upto[wave] = here;
    lds_sync();
    int before = here - sum + waves_below(upto, wave);
    if (before < rest && rest <= before + sum) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (before < rest && rest <= before + c[i]) {
          digit = uint32_t(top - i);
          left = rest - before;
        }
        before += c[i];
      }
    }
    lds_sync();
    rest = left;
    return digit;
  }
};

// Rows of a sequence and head.
struct Place {
  const KvEvictParams& p;
  int b, kh;
  // Row of token t.
  __device__ __forceinline__ uint32_t row(int t) const {
    const int page = int(p.by_page(unsigned(t)));
    const unsigned entry = min(unsigned(p.table[int64_t(b) * p.width + page]), unsigned(p.pages - 1));
    return (entry * unsigned(p.hk) + unsigned(kh)) * unsigned(p.page) + unsigned(t - page * p.page);
  }
};

// Batches first, first + step, ... of `moves` rows from one place to another by a block
// of `threads`: 2^row_shift threads have a key's units, then a value's (and a part of
// either's exponents), four moves at a time.  places(move, to, from) gives the rows.
// IN_ORDER: rows may overlap their new places; a lower move's row is read before a
// higher one's is written, and all threads come along.
template <bool IN_ORDER, class U, class E, class Places>
__device__ __forceinline__ void copy_rows(const KvEvictParams& p, E* k_exps, E* v_exps, int exp_units, int threads, int moves, int first,
                                          int step, Places places) {
  const int units = p.row_bytes / int(sizeof(U)), lanes = 1 << p.row_shift, u0 = int(threadIdx.x) & (lanes - 1);
  const int per = threads >> p.row_shift, mine = int(threadIdx.x) >> p.row_shift;
  for (int64_t i0 = int64_t(first) * 4 * per; i0 < moves; i0 += int64_t(step) * 4 * per) {
    uint32_t to[4], from[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t i = i0 + e * per + mine;
      if (i < moves) places(int(i), &to[e], &from[e]);
    }
    // (One turn but for rows of over 32 units.)
    for (int u = u0; IN_ORDER ? u - u0 < 2 * units : u < 2 * units; u += lanes) {
      U* rows = static_cast<U*>(u < units ? p.k_cache : p.v_cache);
      E* exps = u < units ? k_exps : v_exps;
      const int v = u < units ? u : u - units;
      U x[4];
      E y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (u < 2 * units && i0 + e * per + mine < moves) {
          x[e] = rows[int64_t(from[e]) * units + v];
          if (v < exp_units) y[e] = exps[int64_t(from[e]) * exp_units + v];
        }
      if (IN_ORDER) __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (u < 2 * units && i0 + e * per + mine < moves) {
          rows[int64_t(to[e]) * units + v] = x[e];
          if (v < exp_units) exps[int64_t(to[e]) * exp_units + v] = y[e];
        }
      if (IN_ORDER) __syncthreads();
    }
  }
}
// (The units of exponents are at most as many as a row's: d / 32 bytes or fewer words, and d / 32 units of 16 bytes.)
template <bool IN_ORDER, class U, class Places>
__device__ __forceinline__ void copy_moves(const KvEvictParams& p, int threads, int moves, int first, int step, Places places) {
  if (p.exp_words)
    copy_rows<IN_ORDER, U>(p, reinterpret_cast<uint32_t*>(p.k_exps), reinterpret_cast<uint32_t*>(p.v_exps), p.exp_bytes / 4, threads,
                           moves, first, step, places);
  else
    copy_rows<IN_ORDER, U>(p, p.k_exps, p.v_exps, p.exp_bytes, threads, moves, first, step, places);
}

// The mass of a rank (a NaN for NaN, 0 for -0).
__device__ __forceinline__ float mass_of(uint32_t r) { return __uint_as_float(r == 0u ? 0x7fc00000u : r & 0x80000000u ? r ^ 0x80000000u : ~r); }

constexpr int kBuckets = 1024;      // of the rank's highest 10 bits
// Where the workspace holds what, for each (sequence, head), in 32-bit words.
struct Lists {
  int chunks, chunk;                // tokens a chunk, a multiple of kSelect
  int64_t places;                   // most places that can fall vacant
  int64_t hist, stats, some, vacant, movers, mover_mass, mass, ties, gaps, stride;
};
__host__ __device__ inline Lists lists_of(int64_t keep, int64_t recent, int64_t max_length) {
  Lists l;
  const int64_t a = keep - recent, b = max_length - keep;
  l.places = a < b ? a : b;
  if (l.places < 0) l.places = 0;
  const int64_t least = (max_length + 63) / 64;
  l.chunk = int(((least > 4096 ? least : 4096) + kSelect - 1) / kSelect * kSelect);
  l.chunks = int((max_length + l.chunk - 1) / l.chunk);
  l.hist = 0;
  l.stats = l.hist + int64_t(l.chunks) * kBuckets;    // a chunk's tokens in the bucket, above it below the front, above it from there on
  l.some = l.stats + int64_t(l.chunks) * 4;           // tokens in the bucket, a chunk's from its first token's place on
  l.vacant = l.some + int64_t(l.chunks) * l.chunk;
  l.movers = l.vacant + l.places;
  l.mover_mass = l.movers + l.places;
  l.mass = l.mover_mass + l.places;
  l.ties = l.mass + (keep < max_length ? keep : max_length);
  l.gaps = l.ties + 1;
  l.stride = l.gaps + 1;
  return l;
}

// ---------------------------------------------------------------------------
// Up to 16384 tokens: selected by one block.

// A sequence's tokens are in one block's LDS up to here: 6.2 us for 64 tokens, 0.8 for each 1024
// more.  In chunks over the chip it is the launches' time (40 heads of 16384 tokens, 1639 kept: 30.4
// us with three launches and 35.4 with five; a sequence of 16384 of 4 heads 24.5 and 28.5).
constexpr int kOneTokens = 16384, kWords = kOneTokens / kWave;
// As many moves are made by the same block, which has one compute unit's share of the memory's rate:
// vacant places and `recent` (32 heads of 4096 tokens, 1000 kept: 23.5 us; with two more launches
// and 2000 kept 26.8, where one took 34.7).
constexpr int kFewRows = 1024;
using Top = Digits<4096, 2>;        // of the rank's highest 12 bits: most masses share an octave or two, and
using Low = Digits<1024, 1>;        // additions to one address wait for each other; then two digits of 10

// FEW: the block moves the rows as well; otherwise it leaves lists for evict_move.
template <class U, bool FEW>
__global__ __launch_bounds__(kSelect) void evict_one_kernel(KvEvictParams p) {
  extern __shared__ uint32_t s_rank[];                      // [max_length]
  __shared__ Top s_top;
  __shared__ Low s_low[2];
  // Of 64 tokens each: who is above the border, at it, stays; gaps and movers before them.
  __shared__ uint64_t s_above[kWords], s_equal[kWords];
  __shared__ int s_at[kWords], s_part[2][kWaves];
  __shared__ uint32_t s_to[FEW ? kFewRows : 1], s_from[FEW ? kFewRows : 1];     // tokens, then their rows
  const int kh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = tokens_of(p, b), keep = int(p.keep), recent = int(p.recent), sink = int(p.sink), m = min(n, keep);
  const int64_t head = int64_t(b) * p.hk + kh;
  const float* mass = p.mass + head * p.span;
  int32_t* kept = p.kept + head * p.keep;
  const Lists l = lists_of(p.keep, p.recent, p.max_length);
  uint32_t* ws = static_cast<uint32_t*>(p.workspace) + (FEW ? 0 : head * l.stride);
  // The new masses: in place, or for evict_move.
  float* out = FEW ? p.mass_out + head * p.span : reinterpret_cast<float*>(ws + l.mass);
  if (FEW && kh == 0 && tid == 0) p.lengths_out[b] = m;
  if (n <= keep) {
    for (int64_t j = tid; j < keep; j += kSelect) kept[j] = j < n ? int(j) : -1;
    for (int64_t j = tid; j < (FEW ? p.span : n); j += kSelect) out[j] = j < n ? mass[j] : 0.f;
    return;
  }
  const int end = n - recent, front = keep - recent, want = front - sink;
  s_top.clear();
  s_low[0].clear();
  s_low[1].clear();
  lds_sync();
  // Eight loads under way at once.
  for (int j0 = tid; j0 < n; j0 += 8 * kSelect) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = mass[min(j0 + e * kSelect, n - 1)];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = j0 + e * kSelect;
      const uint32_t r = rank_of(v[e]);
      if (j < n) s_rank[j] = r;
      if (j >= sink && j < end) s_top.add(r >> 20);
    }
  }
  lds_sync();
  uint32_t border = 0u;
  int ties = want;
  if (want > 0) {
    border = s_top.find(ties) << 20;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int shift = 10 - 10 * i;
#pragma unroll 4
      for (int j = sink + tid; j < end; j += kSelect) {
        const uint32_t r = s_rank[j];
        if ((r ^ border) >> (shift + 10) == 0u) s_low[i].add(r >> shift & 1023u);
      }
      lds_sync();
      border |= s_low[i].find(ties) << shift;
    }
  }
  const int words = (end + kWave - 1) / kWave;
  for (int w = wave; w < words; w += kWaves) {
    const int j = w * kWave + lane;
    const uint32_t r = s_rank[min(j, n - 1)];
    const bool here = j < end, inner = here && want > 0 && j >= sink;
    const unsigned long long above = __ballot((here && j < sink) || (inner && r > border)), equal = __ballot(inner && r == border);
    if (lane == 0) {
      s_above[w] = above;
      s_equal[w] = equal;
    }
  }
  lds_sync();
  // A thread a word: the first ties stay too, then gaps below the front and movers from it on, both counts in one number.
  static_assert(kWords <= kSelect, "a thread has one word");
  const uint64_t equal = tid < words ? s_equal[tid] : 0u;
  const int equal_upto = wave_upto(__popcll(equal));
  if (lane == kWave - 1) s_part[0][wave] = equal_upto;
  lds_sync();
  const int left = ties - (equal_upto - __popcll(equal)) - waves_below(s_part[0], wave);
  uint64_t over = equal;                                    // ties that leave
  for (int i = 0; i < left && over != 0u; ++i) over &= over - 1;
  uint64_t stays = 0u;
  int count = 0;
  if (tid < words) {
    auto first = [&](int upto) {                            // the word's tokens below `upto`
      const int k = min(max(upto - tid * kWave, 0), kWave);
      return k == kWave ? ~uint64_t(0) : (uint64_t(1) << k) - 1;
    };
    stays = s_above[tid] | (equal ^ over);
    count = __popcll(first(end) & first(front) & ~stays) | __popcll(stays & ~first(front)) << 16;
  }
  const int upto = wave_upto(count);
  if (lane == kWave - 1) s_part[1][wave] = upto;
  lds_sync();
  int total;
  const int before = upto - count + waves_below(s_part[1], wave, &total);
  total &= 0xffff;
  if (tid < words) {
    s_above[tid] = stays;
    s_at[tid] = before;
  }
  lds_sync();
  int *vacant = reinterpret_cast<int*>(ws + l.vacant), *movers = reinterpret_cast<int*>(ws + l.movers);
  float* mover_mass = reinterpret_cast<float*>(ws + l.mover_mass);
  for (int w = wave; w < words; w += kWaves) {
    const int j = w * kWave + lane, at = s_at[w];
    const bool yes = s_above[w] >> lane & 1u, gap = j < min(end, front) && !yes, go = yes && j >= front;
    const int gap_at = (at & 0xffff) + lanes_below(__ballot(gap)), go_at = (at >> 16) + lanes_below(__ballot(go));
    const uint32_t r = s_rank[min(j, n - 1)];
    if (yes && !go) {
      kept[j] = j;
      out[j] = mass_of(r);
    }
    if constexpr (FEW) {
      if (gap) s_to[gap_at] = j;
      if (go) s_from[go_at] = j;
    } else {
      if (gap) {
        kept[j] = -1;               // until evict_move fills it
        vacant[gap_at] = j;
      }
      if (go) {
        movers[go_at] = j;
        mover_mass[go_at] = mass_of(r);
      }
    }
  }
  if constexpr (!FEW) {
    for (int i = tid; i < recent; i += kSelect) {
      kept[front + i] = end + i;
      out[front + i] = mass_of(s_rank[end + i]);
    }
    if (tid == 0) ws[l.gaps] = uint32_t(total);
    return;
  }
  const int moves = total + recent;
  for (int i = total + tid; i < moves; i += kSelect) {
    s_to[i] = front + i - total;
    s_from[i] = end + i - total;
  }
  lds_sync();
  const Place place = {p, b, kh};
  for (int i = tid; i < moves; i += kSelect) {
    const int to = s_to[i], from = s_from[i];
    kept[to] = from;
    out[to] = mass_of(s_rank[from]);
    s_to[i] = place.row(to);
    s_from[i] = place.row(from);
  }
  for (int64_t j = m + tid; j < p.span; j += kSelect) out[j] = 0.f;
  lds_sync();
  copy_moves<false, U>(p, kSelect, total, 0, 1, [&](int i, uint32_t* to, uint32_t* from) {
    *to = s_to[i];
    *from = s_from[i];
  });
  if (recent == 0) return;
  __syncthreads();
  copy_moves<true, U>(p, kSelect, recent, 0, 1, [&](int i, uint32_t* to, uint32_t* from) {
    *to = s_to[total + i];
    *from = s_from[total + i];
  });
}

// ---------------------------------------------------------------------------
// Longer sequences.

constexpr int kRest = 22 - 11;      // its other bits in two digits of 11
constexpr int kSome = 16384;        // tokens of the bucket that a block has in LDS

// What the blocks of a (sequence, head) share.
struct Chunk {
  Lists l;
  int64_t head;
  int kh, b, n, end, front, sink, want, j0, j1, per, w0, w1;
  const float* mass;
  uint32_t* ws;
  float early[4];

  __device__ __forceinline__ Chunk(const KvEvictParams& p) : l(lists_of(p.keep, p.recent, p.max_length)) {
    kh = blockIdx.y;
    b = blockIdx.z;
    head = int64_t(b) * p.hk + kh;
    n = tokens_of(p, b);
    sink = int(p.sink);
    front = int(p.keep - p.recent);
    want = front - sink;
    end = n > p.keep ? n - int(p.recent) : 0;
    j0 = min(end, int(blockIdx.x) * l.chunk);
    j1 = min(end, j0 + l.chunk);
    mass = p.mass + head * p.span;
    ws = static_cast<uint32_t*>(p.workspace) + head * l.stride;
    // This wave's tokens of the chunk.
    per = l.chunk / kWaves;
    w0 = min(j1, j0 + int(threadIdx.x) / kWave * per);
    w1 = min(j1, w0 + per);
    // The first of them on their way before anything is waited for.
    load(w0, early);
  }

  __device__ __forceinline__ void load(int t, float* m) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = t + e * kWave + int(threadIdx.x) % kWave;
      m[e] = j < w1 ? mass[j] : 0.f;
    }
  }

  // f(token, whether it is one, its mass) for this wave's tokens in order, 64 at a time and all
  // lanes together.
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    const int lane = threadIdx.x % kWave;
    for (int t = w0; t < w1; t += 4 * kWave) {
      float m[4] = {early[0], early[1], early[2], early[3]};
      if (t != w0) load(t, m);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t + e * kWave < w1) f(t + e * kWave + lane, t + e * kWave + lane < w1, m[e]);
    }
  }
};

__global__ __launch_bounds__(kSelect) void evict_count_kernel(KvEvictParams p) {
  __shared__ Digits<kBuckets, 2> s_top;
  const Chunk c(p);
  const int tid = threadIdx.x;
  if (c.end == 0) return;
  s_top.clear();
  lds_sync();
  c.each([&](int j, bool here, float m) {
    if (here && j >= c.sink) s_top.add(rank_of(m) >> 22);
  });
  lds_sync();
  c.ws[c.l.hist + int64_t(blockIdx.x) * kBuckets + tid] = uint32_t(s_top.count[2 * tid] + s_top.count[2 * tid + 1]);
}

__global__ __launch_bounds__(kSelect) void evict_bucket_kernel(KvEvictParams p) {
  __shared__ Digits<kBuckets, 1> s_top;
  __shared__ int s_part[3][kWaves];
  const Chunk c(p);
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  if (c.end == 0 || c.want == 0) return;
  int sum = 0;
#pragma unroll 16
  for (int i = 0; i < c.l.chunks; ++i) sum += int(c.ws[c.l.hist + int64_t(i) * kBuckets + tid]);
  s_top.count[tid] = sum;
  lds_sync();
  int ties = c.want;
  const uint32_t bucket = s_top.find(ties);
  int in = 0, low = 0, high = 0;
  c.each([&](int j, bool here, float m) {
    here = here && j >= c.sink;
    const uint32_t top = rank_of(m) >> 22;
    in += __popcll(__ballot(here && top == bucket));
    low += __popcll(__ballot(here && top > bucket && j < c.front));
    high += __popcll(__ballot(here && top > bucket && j >= c.front));
  });
  if (lane == 0) {
    s_part[0][wave] = in;
    s_part[1][wave] = low;
    s_part[2][wave] = high;
  }
  lds_sync();
  int at = waves_below(s_part[0], wave);
  uint32_t* some = c.ws + c.l.some + c.j0;
  c.each([&](int j, bool here, float m) {
    const uint32_t r = rank_of(m);
    const bool yes = here && j >= c.sink && r >> 22 == bucket;
    const unsigned long long all = __ballot(yes);
    // The rank's other 22 bits, and whether it is below the front.
    if (yes) some[at + lanes_below(all)] = (r & 0x3fffffu) | uint32_t(j < c.front) << 31;
    at += __popcll(all);
  });
  if (wave < 4) {
    int x = int(bucket);
    if (wave < 3) waves_below(s_part[wave], 0, &x);
    if (lane == 0) c.ws[c.l.stats + int64_t(blockIdx.x) * 4 + wave] = uint32_t(x);
  }
  // (Every block finds the same; the first leaves it.)
  if (blockIdx.x == 0 && tid == 0) c.ws[c.l.ties] = uint32_t(ties);
}

__global__ __launch_bounds__(kSelect) void evict_border_kernel(KvEvictParams p) {
  __shared__ Digits<2048, 2> s_low_digits;
  __shared__ uint32_t s_some[kSome];
  __shared__ int s_equal[64], s_low[64], s_high[64], s_equal_low[64];
  __shared__ int s_wave[4][kWaves];
  const Chunk c(p);
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  int32_t* kept = p.kept + c.head * p.keep;
  float* fresh = reinterpret_cast<float*>(c.ws + c.l.mass);
  if (c.end == 0) {
    // All stay.
    for (int64_t j = int64_t(blockIdx.x) * kSelect + tid; j < p.keep; j += int64_t(gridDim.x) * kSelect) {
      kept[j] = j < c.n ? int(j) : -1;
      if (j < c.n) fresh[j] = c.mass[j];
    }
    return;
  }
  // Lane k has chunk k.
  const int k_mine = min(lane, c.l.chunks - 1);
  int ties = 0, count = 0, above_low = 0, above_high = 0, before = 0;
  uint32_t border = 0u;
  if (c.want > 0) {
    const uint32_t* stats = c.ws + c.l.stats + k_mine * 4;
    count = lane < c.l.chunks ? int(stats[0]) : 0;
    above_low = int(stats[1]);
    above_high = int(stats[2]);
    const uint32_t bucket = stats[3];
    ties = int(c.ws[c.l.ties]);
    // The tokens in the bucket, in LDS where it has room for all.
    const int upto = wave_upto(count);
    before = upto - count;
    const bool fits = __builtin_amdgcn_readlane(upto, kWave - 1) <= kSome;
    if (fits) {
      for (int k = wave; k < c.l.chunks; k += kWaves) {
        const int n = __builtin_amdgcn_readlane(count, k), at = __builtin_amdgcn_readlane(before, k);
        const uint32_t* some = c.ws + c.l.some + int64_t(k) * c.l.chunk;
#pragma unroll 4
        for (int i = lane; i < n; i += kWave) s_some[at + i] = some[i];
      }
    }
    // f(chunk, its tokens in the bucket, how many): a wave takes every 16th chunk.
    auto each_some = [&](auto f) {
      for (int k = wave; k < c.l.chunks; k += kWaves) {
        const int n = __builtin_amdgcn_readlane(count, k);
        if (fits) f(k, s_some + __builtin_amdgcn_readlane(before, k), n);
        else f(k, c.ws + c.l.some + int64_t(k) * c.l.chunk, n);
      }
    };
    uint32_t low = 0u;
#pragma unroll 1
    for (int shift = kRest; shift >= 0; shift -= kRest) {
      s_low_digits.clear();
      lds_sync();
      each_some([&](int, const uint32_t* some, int n) {
#pragma unroll 4
        for (int i = lane; i < n; i += kWave) {
          const uint32_t r = some[i] & 0x3fffffu;
          if (shift == kRest || r >> kRest == low >> kRest) s_low_digits.add(r >> shift & 2047u);
        }
      });
      lds_sync();
      low |= s_low_digits.find(ties) << shift;
    }
    border = bucket << 22 | low;
    // Each chunk's tokens at the border and above it.
    each_some([&](int k, const uint32_t* some, int n) {
      int equal = 0, equal_low = 0, more_low = 0, more_high = 0;
      for (int i0 = 0; i0 < n; i0 += kWave) {
        const bool here = i0 + lane < n;
        const uint32_t v = here ? some[i0 + lane] : 0u, r = v & 0x3fffffu;
        const bool below = v >> 31 != 0u;
        equal += __popcll(__ballot(here && r == low));
        equal_low += __popcll(__ballot(here && r == low && below));
        more_low += __popcll(__ballot(here && r > low && below));
        more_high += __popcll(__ballot(here && r > low && !below));
      }
      if (lane == 0) {
        s_equal[k] = equal;
        s_equal_low[k] = equal_low;
        s_low[k] = more_low;
        s_high[k] = more_high;
      }
    });
  } else if (tid < c.l.chunks) {
    s_equal[tid] = s_equal_low[tid] = s_low[tid] = s_high[tid] = 0;
  }
  lds_sync();
  // Up to this chunk: ties, vacant places, movers.  And all vacant places.
  int tie0, gap0, go0, gaps;
  {
    const int k = k_mine, a = k * c.l.chunk, z = min(c.front, min(c.end, a + c.l.chunk));
    const int equal = lane < c.l.chunks ? s_equal[k] : 0, before = wave_upto(equal) - equal;
    const int taken = min(max(ties - before, 0), equal), taken_low = min(taken, s_equal_low[k]);
    const int sinks = min(max(c.sink - a, 0), c.l.chunk);
    const int gap = lane < c.l.chunks ? max(z - a, 0) - (sinks + above_low + s_low[k] + taken_low) : 0;
    const int go = above_high + s_high[k] + taken - taken_low;
    const int gaps_upto = wave_upto(gap), go_upto = wave_upto(go), me = int(blockIdx.x);
    tie0 = __builtin_amdgcn_readlane(before, me);
    gap0 = __builtin_amdgcn_readlane(gaps_upto - gap, me);
    go0 = __builtin_amdgcn_readlane(go_upto - go, me);
    gaps = __builtin_amdgcn_readlane(gaps_upto, kWave - 1);
  }
  // Then up to this wave, from each wave's tokens at the border and above it.
  int equal = 0, equal_low = 0, more_low = 0, more_high = 0;
  c.each([&](int j, bool here, float m) {
    const uint32_t r = rank_of(m);
    const bool inner = here && c.want > 0 && j >= c.sink, above = here && (j < c.sink || (inner && r > border));
    equal += __popcll(__ballot(inner && r == border));
    equal_low += __popcll(__ballot(inner && r == border && j < c.front));
    more_low += __popcll(__ballot(above && j < c.front));
    more_high += __popcll(__ballot(above && j >= c.front));
  });
  if (lane == 0) {
    s_wave[0][wave] = equal;
    s_wave[1][wave] = equal_low;
    s_wave[2][wave] = more_low;
    s_wave[3][wave] = more_high;
  }
  lds_sync();
  {
    // Lane w has wave w.
    const int w = lane % kWaves, a = min(c.j1, c.j0 + w * c.per), z = max(a, min(c.front, min(c.j1, a + c.per)));
    const int n = lane < kWaves ? s_wave[0][w] : 0, seen = tie0 + wave_upto(n) - n;
    const int taken = min(max(ties - seen, 0), n), taken_low = min(taken, s_wave[1][w]);
    const int gap = lane < kWaves ? z - a - s_wave[2][w] - taken_low : 0, go = lane < kWaves ? s_wave[3][w] + taken - taken_low : 0;
    tie0 = __builtin_amdgcn_readlane(seen, wave);
    gap0 += __builtin_amdgcn_readlane(wave_upto(gap) - gap, wave);
    go0 += __builtin_amdgcn_readlane(wave_upto(go) - go, wave);
  }
  int *vacant = reinterpret_cast<int*>(c.ws + c.l.vacant), *movers = reinterpret_cast<int*>(c.ws + c.l.movers);
  float* mover_mass = reinterpret_cast<float*>(c.ws + c.l.mover_mass);
  c.each([&](int j, bool here, float m) {
    const uint32_t r = rank_of(m);
    const bool inner = here && c.want > 0 && j >= c.sink, tie = inner && r == border;
    const unsigned long long all_ties = __ballot(tie);
    const bool yes = here && (j < c.sink || (inner && r > border) || (tie && tie0 + lanes_below(all_ties) < ties));
    const bool gap = here && !yes && j < c.front, go = yes && j >= c.front;
    const unsigned long long all_gaps = __ballot(gap), all_go = __ballot(go);
    tie0 += __popcll(all_ties);
    if (yes && !go) {
      kept[j] = j;
      fresh[j] = m;
    }
    if (gap) {
      kept[j] = -1;                 // until evict_move fills it
      vacant[gap0 + lanes_below(all_gaps)] = j;
    }
    if (go) {
      const int at = go0 + lanes_below(all_go);
      movers[at] = j;
      mover_mass[at] = m;
    }
    gap0 += __popcll(all_gaps);
    go0 += __popcll(all_go);
  });
  for (int i = int(blockIdx.x) * kSelect + tid; i < p.recent; i += int(gridDim.x) * kSelect) {
    kept[c.front + i] = c.end + i;
    fresh[c.front + i] = c.mass[c.end + i];
  }
  if (blockIdx.x == 0 && tid == 0) c.ws[c.l.gaps] = uint32_t(gaps);
}

template <class U>
__global__ __launch_bounds__(256) void evict_move_kernel(KvEvictParams p, int mass_blocks) {
  const int kh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int64_t head = int64_t(b) * p.hk + kh;
  const Lists l = lists_of(p.keep, p.recent, p.max_length);
  const uint32_t* ws = static_cast<const uint32_t*>(p.workspace) + head * l.stride;
  const int n = tokens_of(p, b), m = min(int64_t(n), p.keep), gaps = n > m ? int(ws[l.gaps]) : 0;
  const int *vacant = reinterpret_cast<const int*>(ws + l.vacant), *movers = reinterpret_cast<const int*>(ws + l.movers);
  const float *mover_mass = reinterpret_cast<const float*>(ws + l.mover_mass), *fresh = reinterpret_cast<const float*>(ws + l.mass);
  float* mass = p.mass_out + head * p.span;
  int32_t* kept = p.kept + head * p.keep;
  const int front = n > m ? int(p.keep - p.recent) : m;
  // The first blocks have the masses, the others the rows.
  if (int(blockIdx.x) < mass_blocks) {
    const int first = int(blockIdx.x) * 256 + tid, step = mass_blocks * 256;
#pragma unroll 4
    for (int64_t j = first; j < p.span; j += step) {
      // A vacant place's mass comes below.
      if (j >= front || kept[j] == j) mass[j] = j < m ? fresh[j] : 0.f;
    }
#pragma unroll 2
    for (int i = first; i < gaps; i += step) {
      mass[vacant[i]] = mover_mass[i];
      kept[vacant[i]] = movers[i];
    }
    if (kh == 0 && first == 0) p.lengths_out[b] = m;
    return;
  }
  const Place place = {p, b, kh};
  copy_moves<false, U>(p, 256, gaps, int(blockIdx.x) - mass_blocks, int(gridDim.x) - mass_blocks, [&](int i, uint32_t* to, uint32_t* from) {
    *to = place.row(vacant[i]);
    *from = place.row(movers[i]);
  });
}

template <class U>
__global__ __launch_bounds__(kSelect) void evict_shift_kernel(KvEvictParams p) {
  const int n = tokens_of(p, blockIdx.z), keep = int(p.keep), recent = int(p.recent);
  if (n <= keep) return;
  const Place place = {p, int(blockIdx.z), int(blockIdx.y)};
  auto places = [&](int i, uint32_t* to, uint32_t* from) {
    *to = place.row(keep - recent + i);
    *from = place.row(n - recent + i);
  };
  // Rows that do not overlap their new places are any block's.
  if (n - keep >= recent) copy_moves<false, U>(p, kSelect, recent, blockIdx.x, gridDim.x, places);
  else if (blockIdx.x == 0) copy_moves<true, U>(p, kSelect, recent, 0, 1, places);
}

// Whether one launch does it all.
bool few_rows(int64_t keep, int64_t recent, int64_t max_length) {
  return max_length <= keep || (max_length <= kOneTokens && lists_of(keep, recent, max_length).places + recent <= kFewRows);
}

template <class U>
hipError_t launch(const KvEvictParams& p, hipStream_t stream) {
  const bool few = few_rows(p.keep, p.recent, p.max_length);
  const size_t ranks = p.max_length <= p.keep ? 0 : size_t(p.max_length) * sizeof(uint32_t);
  if (few) {
    evict_one_kernel<U, true><<<dim3(unsigned(p.hk), unsigned(p.batch)), dim3(kSelect), ranks, stream>>>(p);
    return hipGetLastError();
  }
  const Lists l = lists_of(p.keep, p.recent, p.max_length);
  const dim3 grid(unsigned(l.chunks), unsigned(p.hk), unsigned(p.batch));
  if (p.max_length <= kOneTokens) {
    evict_one_kernel<U, false><<<dim3(unsigned(p.hk), unsigned(p.batch)), dim3(kSelect), ranks, stream>>>(p);
  } else {
    if (p.keep > p.recent + p.sink) {
      evict_count_kernel<<<grid, dim3(kSelect), 0, stream>>>(p);
      evict_bucket_kernel<<<grid, dim3(kSelect), 0, stream>>>(p);
    }
    evict_border_kernel<<<grid, dim3(kSelect), 0, stream>>>(p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Enough blocks for four moves a thread, or 2048 masses a block.
  const int64_t heads = int64_t(p.hk) * p.batch;
  auto blocks_of = [&](int64_t want) { return unsigned(std::max<int64_t>(1, std::min<int64_t>(want, std::max<int64_t>(1, 8192 / heads)))); };
  auto moves_of = [&](int64_t moves, int threads) { return ((moves << p.row_shift) + 4 * threads - 1) / (4 * threads); };
  const unsigned masses = blocks_of((p.span + 2047) / 2048), move = masses + (l.places ? blocks_of(moves_of(l.places, 256)) : 0u);
  evict_move_kernel<U><<<dim3(move, unsigned(p.hk), unsigned(p.batch)), dim3(256), 0, stream>>>(p, int(masses));
  e = hipGetLastError();
  if (e != hipSuccess || p.recent == 0) return e;
  const unsigned shift = blocks_of(moves_of(p.recent, kSelect));
  evict_shift_kernel<U><<<dim3(shift, unsigned(p.hk), unsigned(p.batch)), dim3(kSelect), 0, stream>>>(p);
  return hipGetLastError();
}

// The power of two threads that have a move's 2 * units units, at most a wave.
int shift_of(int units) {
  int s = 1;
  while (s < 6 && (1 << s) < 2 * units) ++s;
  return s;
}

}  // namespace

size_t evict_workspace_bytes(int64_t batch, int64_t hk, int64_t keep, int64_t recent, int64_t max_length) {
  if (few_rows(keep, recent, max_length)) return 0;
  return size_t(batch * hk * lists_of(keep, recent, max_length).stride) * sizeof(uint32_t);
}

hipError_t launch_kv_evict(KvEvictParams p, hipStream_t stream) {
  const int unit = p.row_bytes % 16 == 0 ? 16 : 8;
  p.row_shift = shift_of(p.row_bytes / unit);
  p.exp_words = p.exp_bytes % 4 == 0 && (reinterpret_cast<uintptr_t>(p.k_exps) | reinterpret_cast<uintptr_t>(p.v_exps)) % 4 == 0;
  return unit == 16 ? launch<u32x4>(p, stream) : launch<u32x2>(p, stream);
}

}  // namespace cp
