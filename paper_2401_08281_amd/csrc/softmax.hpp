// Host-side declarations shared by the translation units of libvs_softmax.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.hpp"
#include "store.hpp"

// A launch of n workgroups: in two dimensions from 2^23 on, since HIP drops, without an error, what goes beyond 2^32
// threads of one dimension.  The workgroups past the n-th have nothing to do.
constexpr int64_t kGroupsInRow = (int64_t)1 << 23;
inline dim3 grid_2d(int64_t n) {
  return n <= kGroupsInRow ? dim3((unsigned)n) : dim3((unsigned)kGroupsInRow, (unsigned)((n + kGroupsInRow - 1) / kGroupsInRow));
}
__device__ __forceinline__ int64_t group_id() { return blockIdx.x + (int64_t)gridDim.x * blockIdx.y; }

// ---- what the kernels of both files share ------------------------------------------
constexpr float kLog2e = 1.44269504088896340736f;
// (the same in all lanes, and known to be: what follows from it is scalar)
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
// e^t for t <= 0 (v_exp_f32: one unit in the last place, results below 2^-126 flush to 0 or a denormal, both fine here)
__device__ __forceinline__ float exp_neg(float t) { return __builtin_amdgcn_exp2f(t * kLog2e); }
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) v += __shfl_xor(v, w);
  return v;
}
// The exponent of the power of two that brings a largest component of `mx` to [2^14, 2^15), the top of fp16's range: what lies
// 2^28 below it still has its head's full 11 bits, and half a step of the smallest numbers, 2^-25, is 2^-39 of the largest
// component.  A head and a tail together keep 2^-24 of a component, as fp32 does, down to 2^-15 of the largest.
__device__ __forceinline__ int top_exponent(float mx) {
  const int e = mx > 0.f && mx < __builtin_inff() ? 15 - (int)__builtin_amdgcn_frexp_expf(mx) : 0;
  return e < -126 ? -126 : (e > 126 ? 126 : e);
}
// The end of a loop body whose last matrix instructions' results may be read right behind the loop: the hardware does
// not wait for them, and the compiler, which counts the wait states in between, has left them out where it copied an
// accumulator at the start of the block behind the loop (v_accvgpr_read one instruction after the product: a stale
// value).  A 32x32x16 product's 8 passes are over after 12 wait states, any other one's here after fewer than 20.
__device__ __forceinline__ void settle_products() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// ---- log-probabilities over rows (kernels_logprob.hip) ---------------------------
// A matrix as the matrix cores read it: rows of whole 128-byte K blocks (two units of 64 bytes), `rows` of them that
// exist.  A K unit holds 32 fp16 or bf16 elements, or (planes == 2) 16 fp16 heads and behind them their 16 fp16 tails.
// scale: factor of every row (a power of two), or null (ones).
struct SmMatrix {
  const void* p = nullptr;
  int64_t row_bytes = 0;
  int64_t rows = 0;
  const float* scale = nullptr;
};
constexpr int kSmTileRows = 256;    // rows and queries that a workgroup takes
constexpr int kSmTileQueries = 128;
constexpr int kSmRecRows = 128;     // rows that a softmax record covers
constexpr int kSmFewQueries = 64;   // up to here the rows are streamed past all queries

struct SmForm {                     // how the rows of a type are multiplied
  int dtype, planes;                // planes 2: fp32 as head and tail
  int per_block() const { return planes == 2 ? 32 : 64; }
  int64_t blocks(int64_t k) const { return (k + per_block() - 1) / per_block(); }
};

// A matrix [n, d] to be prepared; two go in one launch (n = 0: none).
struct SmSide {
  const void* x = nullptr;
  int64_t n = 0;
  const float* bias = nullptr;      // rows whose bias is -inf become zeros
  const float* factor = nullptr;    // of every row, for its columns; a row of factor 0 is not read
  void* rows = nullptr;             // out: every row as K blocks of fp16 parts times 1 / row_scale, its largest component in
  float* row_scale = nullptr;       // [2^14, 2^15); infinite or NaN as its largest component is
  void* cols = nullptr;             // out: every column of (factor x) as K blocks over the rows, likewise
  float* col_scale = nullptr;
  u32* colmax = nullptr;            // [d] of scratch, zeros on entry
  int64_t np = 0;                   // (rows in whole K blocks)
};
void launch_sm_prep_rows(const SmForm& f, const SmSide& a, const SmSide& b, int d, hipStream_t st);
void launch_sm_prep_cols(const SmForm& f, const SmSide& a, const SmSide& b, int d, hipStream_t st);

struct SmScores {                   // s = scale <q, x> + bias for rows x0 .. x0 + nx of x
  SmMatrix x, q;
  int64_t kunits = 0;               // K units of a row
  int64_t nx = 0, nq = 0;
  const float* bias = nullptr;      // of these rows
  float scale = 1.f;
  const void* raw_x = nullptr;      // the vectors themselves, where x and q are prepared copies
  const void* raw_q = nullptr;
  int d = 0, dtype = 0;
};
struct SmRecords {                  // softmax of 128 rows: {max, sum, sum e (s - max), second best | position of the max}
  float4* rec = nullptr;            // [nq, parts]
  int64_t parts = 0;
  float* keep = nullptr;            // [nq, keep_ld] the scores themselves, or null (keep_ld: whole tiles of rows)
  int64_t keep_ld = 0;
};
void launch_sm_scores(const SmForm& f, bool direct, const SmScores& s, const SmRecords& r, bool second, hipStream_t st);
void launch_sm_scores_few(int dtype, const void* x, int64_t nb, const void* q, int64_t nq, int d, float scale,
                          const float* bias, const SmRecords& r, bool second, hipStream_t st);
struct SmFinish {
  const void* x; int64_t nb; const void* q; int64_t nq; int d, dtype; float scale; const float* bias;
  const int64_t* targets; int nt, k;
  float* logp; float* lse; float* entropy; float* top_logp; int64_t* top_ids;
};
void launch_sm_finish(const SmFinish& f, const SmRecords& r, hipStream_t st);

// backward
struct SmGrads {
  const float* lse; const float* entropy; const int64_t* targets; int nt;
  const float* g_logp; const float* g_lse; const float* g_entropy;
};
// coef[i] = {coefficient of p, g_entropy, entropy, lse}, bound[i]: a power of two that no |G_ij| exceeds; clear <- zeros
void launch_sm_coefs(const SmGrads& g, int64_t nq, int64_t nb, float4* coef, float* bound, u32* clear, int n_clear, hipStream_t st);
struct SmGOut {
  const float4* coef; const float* bound; const int64_t* targets; int nt; const float* g_logp; int64_t row0;
  void* g; int64_t g_row_bytes;     // [nq][K blocks over the rows], or null
  void* gt; int64_t gt_row_bytes;   // [nx][K blocks over the queries], or null
  float* db; int64_t db_ld;         // [query tiles, db_ld] partial column sums, or null
  bool small;                       // tiles of 128 rows by 64 queries (256 by 128)
};
bool sm_gradients_small(const SmForm& f, int64_t nx, int64_t nq, int64_t kblocks);
void launch_sm_gradients(const SmForm& f, bool direct, const SmScores& s, const SmGOut& o, hipStream_t st);
// out[b][a] (+)= sum_k A[a][k] B[b][k], K blocks split over workgroups: part[split][b][ld]
struct SmProductPlan {
  bool big; int splits;
  int64_t groups;                   // workgroups, of pieces of fewer rows fewer
};
SmProductPlan plan_sm_product(int64_t rows_a, int64_t rows_b, int64_t kblocks);
void launch_sm_product(const SmForm& f, const SmProductPlan& p, const SmMatrix& A, const SmMatrix& B, int64_t kblocks, bool add,
                       float* part, int64_t ld, hipStream_t st);
// out[b][a] = alpha scale_a[a] sum_k A[a][k] B[b][k], in `dtype`; 0 where bias[b] is -inf (bias: or null)
void launch_sm_product_direct(const SmForm& f, const SmMatrix& A, const SmMatrix& B, int64_t kblocks, const float* scale_a,
                              float alpha, const float* bias, int dtype, void* out, hipStream_t st);
// out[b][a] = alpha scale_a[a] scale_b[b] sum_split part[split][b][a], likewise
void launch_sm_product_out(const float* part, int splits, int64_t rows, int64_t ld, int d, const float* scale_a,
                           const float* scale_b, float alpha, const float* bias, int dtype, void* out, hipStream_t st);
void launch_sm_sum_parts(const float* part, int64_t n_parts, int64_t ld, int64_t n, float* out, hipStream_t st);
void launch_sm_zero(void* p, int64_t bytes, hipStream_t st);

// ---- attention over 4-bit codes (kernels_attend.hip) ------------------------------
struct AttendCall {
  const IvfStore* ix;
  const void* q; int64_t nq; int dk, v0, dtype; float scale; const int64_t* limits;
  const int32_t* probes; int nprobe;             // null: all lists
  const float* lse; const void* g_out; const float* g_lse;   // backward
  void* out; float* out_lse;
};
struct AttendPlan {
  int qb, nsplit, nout, lds;                     // queries a workgroup takes; parts of their rows; results; bytes of LDS
  int64_t per, ld;                               // rows (probes) of a part; floats of a partial result
  bool fits;
  bool tiles;                                    // decoded tiles on the matrix cores, in pieces of w components,
  int w, nq16, nb;                               // 16 nq16 queries and up to 64 nb results a workgroup
};
AttendPlan attend_plan(const IvfpqDims& g, int64_t ntotal, int64_t nq, int dk, int v0, int dtype, int nprobe, bool grad);
void launch_attend_pad(const void* q, int64_t nq, int dk, int d, int dtype, float* out, hipStream_t st);
// part: [nq][nsplit][ld] floats of scratch
void launch_attend(const AttendCall& c, const AttendPlan& p, bool grad, float* part, hipStream_t st);
