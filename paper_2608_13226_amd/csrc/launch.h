// Host-side launchers: the only interface between the C-ABI layer (api.hip)
// and the kernel translation units.  Every launcher enqueues on `stream`,
// never synchronises, and returns the HIP status of its launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cp {

// Workspace of coverprune_fst_cost.
struct FstScratch {
  float* inv_norm;                // [n] 1 / |f_i| (0 for a zero row)
  unsigned int* mf_bits;          // max d_f as float bits
  unsigned long long* mx2_bits;   // max squared distance as double bits
  int* tau_min;                   // min frame index
  int* tau_max;                   // max frame index
};

struct FstParams {
  const void* feats;
  bool bf16;
  int n;
  int d;
  const float* pos;
  const int32_t* frame;
  float lambda_f, lambda_x, lambda_tau, kappa;
  float inv_log1p_kappa;          // 1 / log1p(kappa), unused when kappa == 0
  float* cost;                    // [n, n] target-major
  float* maxima;                  // [3] or nullptr
};

hipError_t launch_fst_prep(const FstParams& p, const FstScratch& s, hipStream_t stream);
hipError_t launch_gram(const FstParams& p, const FstScratch& s, hipStream_t stream);
hipError_t launch_fst_epilogue(const FstParams& p, const FstScratch& s, hipStream_t stream);

// The epilogue of coverprune_prune (n a multiple of 64): the cost, and for
// the incremental greedy that follows, its source-major copy T and the
// step-0 gains as partial sums over 64-target blocks.
struct EpiSgs {
  float* T;                       // [n][ldt] T[s][t] = C(s, t)
  int ldt;
  long long* part;                // [n / 64][n] fixed-point partial gains
  const float* v;                 // [n] capacities
  float c0;
  const int* scale;               // the greedy's fixed-point exponent, set before the launch
};
hipError_t launch_fst_epilogue_sgs(const FstParams& p, const FstScratch& s, const EpiSgs& g, hipStream_t stream);

// Greedy selection.
struct SgsParams {
  const float* cost;              // [n, n] target-major
  int n;
  const float* capacity;          // [n]
  int k;
  float c0;
  int32_t* selected;              // [k]
  double* step_gain;              // [k] or nullptr
  double* step_objective;         // [k] or nullptr
  int32_t* assign;                // [n] or nullptr
  void* workspace;
  size_t workspace_bytes;
};

// Dense form.  Up to n = 8192 it asks for the workspace of the incremental
// form too and runs that instead of the sweeps when the data allow it (see
// k_sgs.hip); sgs_sweep_workspace_bytes is what the sweeps alone need.
size_t sgs_workspace_bytes(int64_t n, int64_t k);
size_t sgs_sweep_workspace_bytes(int64_t n, int64_t k);
hipError_t launch_sgs_dense(const SgsParams& p, hipStream_t stream);
// Incremental form: the rows schedule (workspace about 4 n bytes per token)
// unless `compact` or the scene is too large for it, else the exchange
// schedule (about 16 bytes per token).
size_t sgs_inc_workspace_bytes(int64_t n, int64_t k, bool compact);
hipError_t launch_sgs_incremental(const SgsParams& p, bool compact, hipStream_t stream);
// The rows schedule with its data checked on the device; `unfit` stays null
// where it does not serve the scene.  Otherwise words of the workspace: *unfit
// is set when the data are outside the fixed point's domain (the outputs are
// then not written), *tie when an exact gain decided between candidates,
// *abort when the launch gave up; *scale is the grid, 2^-scale.
struct SgsChecked {
  unsigned int* unfit;
  const unsigned int* tie;
  const unsigned int* abort;
  const int* scale;
};
hipError_t launch_sgs_checked(const SgsParams& p, SgsChecked* checked, hipStream_t stream);
// The incremental greedy after launch_fst_epilogue_sgs (coverprune_prune):
// the rows schedule, whose T and step-0 partial gains that epilogue writes.
// sgs_fused_fits: n a multiple of 64 that the rows schedule serves on this
// device.  sgs_fused_prepare points f into p.workspace (sized by
// sgs_fused_workspace_bytes) and enqueues the scale the epilogue needs;
// launch_sgs_fused runs the greedy itself.
struct SgsFused {
  float* T;
  int ldt;
  long long* part;
  int P;
  int* scale;
};
bool sgs_fused_fits(int64_t n);
size_t sgs_fused_workspace_bytes(int64_t n, int64_t k);
hipError_t sgs_fused_prepare(const SgsParams& p, SgsFused* f, hipStream_t stream);
hipError_t launch_sgs_fused(const SgsParams& p, const SgsFused& f, hipStream_t stream);
// Up to 16 scenes in one cooperative launch (incremental form); the scenes'
// workspaces lie one after another in `workspace` (each p[s].workspace is
// ignored).
size_t sgs_inc_batch_workspace_bytes(const int64_t* n, const int64_t* k, int count, bool compact);
hipError_t launch_sgs_incremental_batch(const SgsParams* p, int count, bool compact, void* workspace,
                                        hipStream_t stream);
// Local form: gains over the neighbour table nbr [n, g] (g <= 128, n <= 16384).
size_t sgs_local_workspace_bytes(int64_t n, int64_t k);
hipError_t launch_sgs_local(const SgsParams& p, const int32_t* nbr, int g, hipStream_t stream);

// Latency floor of a greedy step: rounds of the candidate exchange, each
// followed (read_rows) by the read of a row of `rows` [n_rows][row_len] that
// the exchange's winner names.  row_len is a multiple of 256, at most 32768.
size_t step_floor_workspace_bytes();
hipError_t launch_step_floor(const float* rows, int n_rows, int row_len, int rounds, bool read_rows, void* workspace,
                             hipStream_t stream);

// Nearest-neighbour tables: out [n, g], n <= 32768, g <= min(n, 1024).
hipError_t launch_knn(const float* pos, int n, int g, int32_t* out, hipStream_t stream);
// The same tables with scratch space: the tokens in spatial order, whose chunks'
// bounding boxes rule most of them out.  spos [n] (x, y, z, token as bits) is
// left for the caller's use; boxes holds knn_boxes_bytes(n).
size_t knn_boxes_bytes(int64_t n);
hipError_t launch_knn_sorted(const float* pos, int n, int g, int32_t* out, float4* spos, void* boxes,
                             hipStream_t stream);

// The greedy step solved as written: entropic semi-relaxed transport per step.
struct LiteralParams {
  const float* cost;              // [n, n] target-major
  int n;
  const float* capacity;          // [n]
  int k;                          // 1 <= k <= min(n, 4096)
  float epsilon;
  int rounds;
  const int32_t* follow;          // [k] or nullptr
  int32_t* selected;              // [k]
  double* step_score;             // [k] or nullptr
  double* step_residual;          // [k] or nullptr
  double* objective;              // [1] or nullptr
  void* workspace;
  size_t workspace_bytes;
};

// sgs_literal_min_workspace_bytes: what the separate launches need.
size_t sgs_literal_min_workspace_bytes(int64_t n, int64_t k);
size_t sgs_literal_workspace_bytes(int64_t n, int64_t k);
hipError_t launch_sgs_literal(const LiteralParams& p, hipStream_t stream);

// FST capacity.
struct CapacityParams {
  const void* feats;
  bool bf16;
  int n;
  int d;
  const float* pos;
  const int32_t* frame;
  int nn;                         // neighbours per token, 1 <= nn <= n - 1
  float alpha_f, alpha_x, alpha_tau;
  float* capacity;                // [n]
  double* score;                  // [n] or nullptr
  void* workspace;
  size_t workspace_bytes;
};

// With capacity_min_workspace_bytes the tokens stay in index order.
size_t capacity_workspace_bytes(int64_t n, int64_t nn);
size_t capacity_min_workspace_bytes(int64_t n, int64_t nn);
hipError_t launch_capacity(const CapacityParams& p, hipStream_t stream);

// CoverPrune-Lite.
struct LiteParams {
  const void* feats;
  bool bf16;
  int n;
  int d;
  const float* pos;
  const int32_t* frame;
  const float* capacity;
  int k;
  float lambda_f, lambda_x, lambda_tau, kappa;
  double inv_log1p_kappa;
  double grid_scale;              // 256 / voxel_size, float64
  int32_t* selected;              // [k]
  int32_t* group;                 // [n] or nullptr
  double* objective;              // [1] or nullptr
  double* token_cost;             // [n] or nullptr
  void* workspace;
  size_t workspace_bytes;
};

size_t lite_workspace_bytes(int64_t n, int64_t k);
hipError_t launch_lite(const LiteParams& p, hipStream_t stream);

// The serving operators.

// HIP launches less than 2^32 work items a dimension.  A grid of `blocks` blocks
// of `threads` in as many launches as that takes: launch(first block, blocks).
template <class F>
hipError_t launch_blocks(int64_t blocks, int threads, F launch) {
  const int64_t most = ((int64_t(1) << 32) - 1) / threads;
  for (int64_t first = 0; first < blocks; first += most) {
    launch(first, unsigned(blocks - first < most ? blocks - first : most));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

enum class ServeType { kBf16, kF16, kF32, kE4m3, kE2m1 };

struct RmsNormParams {
  const void* x;                  // [rows, d]
  const void* residual;           // [rows, d] or nullptr
  const void* weight;             // [d]
  void* out;                      // [rows, d]
  float* out_scale;               // [rows], with quantize
  void* residual_out;             // [rows, d] with residual
  int64_t rows;                   // 1 <= rows < 2^31
  int d;                          // 1 <= d <= 65536
  float eps;
  ServeType type;                 // of x, residual, weight, residual_out; and of out unless quantize
  bool quantize;                  // out is e4m3
};
hipError_t launch_rms_norm(const RmsNormParams& p, hipStream_t stream);

// y = x (codes - zero) scale over groups of `group` consecutive k.
struct W4Params {
  const void* x;                  // [m, k], `type` or e4m3 (x_scale then set)
  const float* x_scale;           // [m] or nullptr
  const uint8_t* weight;          // [n, k / 2], two codes a byte, the even k low
  const void* scale;              // [n, k / group] `type`
  const uint8_t* zero;            // [n, k / group] or nullptr (8)
  void* y;                        // [m, n]
  int64_t m, n;
  int k, group;                   // k % group == 0, group % 32 == 0, k <= 2^20
  unsigned group_magic;           // r / (group / 32) = (r * magic >> 32) + r * one for r <= 2^15:
  unsigned group_one;             // magic = ceil(2^32 / (group / 32)) and one = 0, or for group 32 0 and 1
  ServeType type;                 // kBf16 or kF16
  ServeType y_type;               // `type` or kF32
};
hipError_t launch_w4_matvec(const W4Params& p, hipStream_t stream);

struct KvAppendParams {
  const void* q;                  // [tokens, hq, d] at token stride q_stride, or nullptr
  const void* k;                  // [tokens, hk, d] at k_stride
  const void* v;                  // [tokens, hk, d] at v_stride
  int64_t q_stride, k_stride, v_stride;   // elements
  const int32_t* positions;       // [tokens]
  const int64_t* slots;           // [tokens]
  const float* inv_freq;          // [rot / 2]
  const float* k_scale;           // [hk] or nullptr, e4m3 caches
  const float* v_scale;
  void* q_out;                    // [tokens, hq, d], with q
  void* k_cache;                  // [pages, hk, page, d]
  void* v_cache;
  int64_t tokens, pages;
  int hq, hk, d, rot, page;
  float magnitude;
  bool interleaved;
  bool cache8;                    // caches are e4m3
  ServeType type;
};
hipError_t launch_kv_append(const KvAppendParams& p, hipStream_t stream);

// n / d for 0 <= n < 2^31 without a division: (2 n * magic >> 32) >> shift, with shift =
// ceil(log2 d) and magic = ceil(2^(31 + shift) / d).
struct Divide {
  unsigned magic = 0, shift = 0;
  Divide() = default;
  explicit Divide(int64_t d) {
    while ((int64_t(1) << shift) < d) ++shift;
    magic = unsigned(((int64_t(1) << (31 + shift)) + d - 1) / d);
  }
  __host__ __device__ unsigned operator()(unsigned n) const { return unsigned(uint64_t(2u * n) * magic >> 32) >> shift; }
};

// The caches of 4 bits: codes two a byte, the even dim low, and exponents of blocks of 32 dims.
struct KvAppend4Params {
  const void* q;                  // [tokens, hq, d] at token stride q_stride, or nullptr
  const void* k;                  // [tokens, hk, d] at k_stride
  const void* v;                  // [tokens, hk, d] at v_stride
  int64_t q_stride, k_stride, v_stride;   // elements
  const int32_t* positions;       // [tokens]
  const int64_t* slots;           // [tokens]
  const float* inv_freq;          // [rot / 2]
  void* q_out;                    // [tokens, hq, d], with q
  uint8_t* k_cache;               // [pages, hk, page, d / 2]
  uint8_t* v_cache;
  uint8_t* k_scale;               // [pages, hk, page, d / 32]
  uint8_t* v_scale;
  int64_t tokens, pages;
  int hq, hk, d, rot, page;       // d % 32 == 0
  Divide by_page, by_runs;        // by d / 8
  double magnitude;
  bool interleaved;
  ServeType type;
};
hipError_t launch_kv_append4(const KvAppend4Params& p, hipStream_t stream);

struct KvGatherParams {
  const void* k_cache;            // [pages, hk, page, d], or d / 2 bytes of codes
  const void* v_cache;
  const void* k_scale;            // e4m3: [hk] float or nullptr; e2m1: [pages, hk, page, d / 32] exponents
  const void* v_scale;
  const int64_t* slots;           // [tokens]
  void* k_out;                    // [tokens, hk, d]
  void* v_out;
  int64_t tokens, pages;
  int hk, d, page;
  Divide by_page;
  ServeType type;                 // of the outputs
  ServeType held;                 // `type`, kE4m3 or kE2m1 (d % 32 == 0)
};
hipError_t launch_kv_gather(const KvGatherParams& p, hipStream_t stream);

struct AttendParams {
  const void* q;                  // [batch, hq, d]
  const void* k_cache;            // [pages, hk, page, d], or d / 2 bytes of codes
  const void* v_cache;
  const int32_t* table;           // [batch, width]
  const int32_t* lengths;         // [batch]
  const float* k_scale;           // [hk] or nullptr, e4m3 caches
  const float* v_scale;
  const uint8_t* k_exps;          // [pages, hk, page, d / 32], e2m1 caches
  const uint8_t* v_exps;
  void* out;                      // [batch, hq, d]
  float* lse;                     // [batch, hq] or nullptr
  float* mass;                    // [batch, hk, mass_span], launch_attend_mass and launch_attend4_mass
  int64_t mass_span;              // >= max_length
  int64_t pages;                  // pages * hk * page < 2^32
  int64_t max_length;             // 1 <= max_length <= width * page < 2^31
  int batch, hq, hk, d, page, width;
  unsigned page_magic, page_shift;  // t / page = (2 t * magic >> 32) >> shift for 0 <= t < 2^31:
                                  // shift = ceil(log2 page), magic = ceil(2^(31 + shift) / page)
  int window;                     // 0: none
  float scale;
  ServeType type;
  ServeType held;                 // `type`, kE4m3 or (launch_attend4, launch_attend4_mass) kE2m1
  void* workspace;
};
// 0 where one launch writes the result.
size_t attend_workspace_bytes(int64_t batch, int64_t hq, int64_t hk, int64_t d, int64_t max_length, int64_t window, bool mass, bool four);
// Whether HIP launches as many blocks as the join of the runs takes.
bool attend_fits(int64_t batch, int64_t hq, int64_t hk, int64_t d, int64_t max_length, int64_t window, bool mass, bool four);
hipError_t launch_attend(const AttendParams& p, hipStream_t stream);
hipError_t launch_attend4(const AttendParams& p, hipStream_t stream);
hipError_t launch_attend_mass(const AttendParams& p, hipStream_t stream);
hipError_t launch_attend4_mass(const AttendParams& p, hipStream_t stream);

struct KvEvictParams {
  void* k_cache;                  // [pages, hk, page] rows of row_bytes
  void* v_cache;
  uint8_t* k_exps;                // [pages, hk, page] rows of exp_bytes (e2m1), or nullptr
  uint8_t* v_exps;
  const int32_t* table;           // [batch, width]
  const int32_t* lengths;         // [batch]
  const float* mass;              // [batch, hk, span]
  float* mass_out;                // [batch, hk, span], may be mass
  int32_t* kept;                  // [batch, hk, keep]
  int32_t* lengths_out;           // [batch], not lengths
  int64_t span, pages, max_length;  // 1 <= max_length <= min(span, width * page) < 2^31
  int64_t keep, recent, sink;     // 1 <= keep < 2^31, 0 <= sink + recent <= keep
  int batch, hk, page, width;
  Divide by_page;
  int row_bytes, exp_bytes;       // row_bytes a multiple of 8; exp_bytes 0 without exponents
  int row_shift;                  // these two are launch_kv_evict's
  bool exp_words;
  void* workspace;
};
size_t evict_workspace_bytes(int64_t batch, int64_t hk, int64_t keep, int64_t recent, int64_t max_length);
hipError_t launch_kv_evict(KvEvictParams p, hipStream_t stream);

}  // namespace cp
