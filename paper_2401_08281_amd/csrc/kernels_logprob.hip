// Softmax over the rows of a matrix: scores on the matrix cores with the softmax statistics in the
// epilogue (the nq x nb scores are never stored), and the gradients, which compute them again.
//
// Orientation.  Rows of x are operand A of a tile, queries operand B: in the accumulators of
// v_mfma_f32_32x32x16 a lane then holds ONE query (column = lane & 31) and 16 rows per block
// (row = (r & 3) + 8 (r >> 2) + 4 (lane >> 5)), so maxima and sums over rows are register arithmetic with a single
// exchange between lane and lane ^ 32.
#include "../../include/vs_softmax.h"
#include "common.hpp"
#include "softmax.hpp"

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// One score t below the maximum of its group: its weight into l, weight times t into h.  Scores of -inf weigh nothing; a
// NaN stays one in l.
__device__ __forceinline__ void softmax_add(float t, float* l, float* h) {
  const float e = exp_neg(t);
  *l += e;
  *h = __builtin_fmaf(e, fmaxf(t, -1000.f), *h);
}
// Group (m, l, h) under the maximum `top` of several groups.  A group without rows has l = 0 (or NaN).
__device__ __forceinline__ void softmax_join(float top, float m, float gl, float gh, float* l, float* h) {
  if (m == -__builtin_inff()) { *l += gl; return; }
  const float t = m - top, e = exp_neg(t);
  *l = __builtin_fmaf(gl, e, *l);
  if (e > 0.f) *h = __builtin_fmaf(e, __builtin_fmaf(gl, t, gh), *h);
}

template <int DT> struct Elem;
template <> struct Elem<0> { typedef float T; };
template <> struct Elem<1> { typedef _Float16 T; };
template <> struct Elem<2> { typedef __bf16 T; };

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

// ---- tiles -------------------------------------------------------------------------
// A workgroup of four wavefronts takes 256 rows by 128 queries, a wavefront 128 x 64 of them: 12 fragment reads from LDS
// feed 16 products (64 x 64 needs 16).  One K unit (64 bytes) of the 384 operand rows is a stage of 24 KB; two stages
// alternate, the next is requested straight into LDS (global_load_lds_dwordx4) before the products of the present one,
// and two workgroups a CU fill each other's waits and run one's epilogue beside the other's products.  A row's four 16-byte
// pieces are stored at piece ^ ((row >> 2) & 3): a fragment read (32 rows x 2 pieces) then touches every bank evenly.
// With two planes a unit holds 16 heads and their 16 tails, and one stage feeds hi*hi + hi*lo + lo*hi.
// Against tiles of 128 x 128 by 64 x 64 (K units of 128 bytes): bf16 4096 x 65,536 x 768 with its finish 579 us for 616,
// fp32 1000 x 200,003 x 100 348 for 417.
// Products and gradients of few tiles take 128 x 64 by 64 x 32 instead (IB, JB: 32-row and 32-query blocks of a wavefront).
constexpr int kTileA = 256, kTileB = 128;
template <int IB, int JB>
constexpr int tile_lds() { return 2 * 64 * (IB + JB) * 64; }

template <int PLANES, bool BF16, int IB = 4, int JB = 2>
struct TileMul {
  static constexpr int TA = 64 * IB, TB = 64 * JB, kStage = (TA + TB) * 64;
  // The products with tails are summed apart where registers allow: added to the large sums one by one, each would leave a
  // rounding of theirs (the gradient of a sharp softmax is what such roundings leave of 1 - p).
  static constexpr bool kApart = PLANES == 2 && IB * JB <= 2;
  static __device__ __forceinline__ f32x16 mul(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (BF16)
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  // acc[ib][jb] of this wavefront: rows 32 (IB wa + ib) .., queries 32 (JB wb + jb) ..; K units [ku0, ku1), at least one
  static __device__ __forceinline__ void run(const SmMatrix& A, int64_t a0, const SmMatrix& B, int64_t b0, int64_t ku0,
                                             int64_t ku1, char* lds, f32x16 (&acc)[IB][JB]) {
    const int lane = lane_id(), wave = wave_id();
    const int wa = wave & 1, wb = wave >> 1;
    // rows past the last one repeat it: their results are dropped
    const char* pa = static_cast<const char*>(A.p) + a0 * A.row_bytes;
    const char* pb = static_cast<const char*>(B.p) + b0 * B.row_bytes;
    const int ra_max = (int)(A.rows - 1 - a0 < TA ? A.rows - 1 - a0 : TA - 1);
    const int rb_max = (int)(B.rows - 1 - b0 < TB ? B.rows - 1 - b0 : TB - 1);
    const char* ga[IB];
    const char* gb[JB];
    const int piece = (lane & 3) ^ ((lane >> 4) & 3);
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      const int r = (wave * IB + i) * 16 + (lane >> 2);
      ga[i] = pa + (int64_t)(r < ra_max ? r : ra_max) * A.row_bytes + ku0 * 64 + piece * 16;
    }
#pragma unroll
    for (int i = 0; i < JB; ++i) {
      const int r = (wave * JB + i) * 16 + (lane >> 2);
      gb[i] = pb + (int64_t)(r < rb_max ? r : rb_max) * B.row_bytes + ku0 * 64 + piece * 16;
    }
    auto request = [&](int stage) {
      char* to = lds + stage * kStage;
#pragma unroll
      for (int i = 0; i < IB; ++i) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)ga[i],
                                         (__attribute__((address_space(3))) void*)(to + (wave * IB + i) * 1024), 16, 0, 0);
        ga[i] += 64;
      }
#pragma unroll
      for (int i = 0; i < JB; ++i) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)gb[i],
                                         (__attribute__((address_space(3))) void*)(to + TA * 64 + (wave * JB + i) * 1024), 16, 0, 0);
        gb[i] += 64;
      }
    };
    const int ra = (wa * 32 * IB + (lane & 31)) * 64, rb = TA * 64 + (wb * 32 * JB + (lane & 31)) * 64, half = lane >> 5, sw = (lane >> 2) & 3;
    request(0);
    const int n = (int)(ku1 - ku0);
    f32x16 low[kApart ? IB : 1][kApart ? JB : 1] = {};
    for (int t = 0; t < n; ++t) {
      __syncthreads();                                  // the stage has landed, the other one is free
      const char* s = lds + (t & 1) * kStage;
      u32x4 a[2][IB], b[2][JB];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int off = ((2 * ks + half) ^ sw) * 16;
#pragma unroll
        for (int ib = 0; ib < IB; ++ib) a[ks][ib] = *reinterpret_cast<const u32x4*>(s + ra + ib * 32 * 64 + off);
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) b[ks][jb] = *reinterpret_cast<const u32x4*>(s + rb + jb * 32 * 64 + off);
      }
      if (t + 1 < n) request((t + 1) & 1);
      auto products = [&](const u32x4 (&fa)[IB], const u32x4 (&fb)[JB]) {
#pragma unroll
        for (int ib = 0; ib < IB; ++ib)
#pragma unroll
          for (int jb = 0; jb < JB; ++jb) acc[ib][jb] = mul(fa[ib], fb[jb], acc[ib][jb]);
      };
      products(a[0], b[0]);
      if constexpr (PLANES == 1) {
        products(a[1], b[1]);
      } else if constexpr (kApart) {
#pragma unroll
        for (int ib = 0; ib < IB; ++ib)
#pragma unroll
          for (int jb = 0; jb < JB; ++jb) {
            low[ib][jb] = mul(a[0][ib], b[1][jb], low[ib][jb]);
            low[ib][jb] = mul(a[1][ib], b[0][jb], low[ib][jb]);
          }
        settle_products();
      } else {
        products(a[0], b[1]);
        products(a[1], b[0]);
      }
    }
    __syncthreads();                                    // LDS is free for the epilogue
    if constexpr (kApart) {
#pragma unroll
      for (int ib = 0; ib < IB; ++ib)
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) acc[ib][jb] += low[ib][jb];
    }
  }
};

// Workgroup number -> tile.  Workgroups go round the 8 XCDs; every XCD takes a contiguous run of tiles, column blocks of
// 8 x 8 tiles inside it, so that the operands of the tiles in flight on one XCD meet in its L2.
__device__ __forceinline__ void tile_of(int64_t wg, int64_t ta, int64_t tb, int64_t* a, int64_t* b) {
  const int64_t n = ta * tb, per = (n + 7) / 8, big = n % 8 == 0 ? 8 : n % 8;   // XCDs with `per` tiles, others per - 1
  const int64_t xcd = wg & 7, i = wg >> 3;
  int64_t t = xcd < big ? xcd * per + i : big * per + (xcd - big) * (per - 1) + i;
  const int64_t strip = 8 * tb;                         // strips of 8 row tiles
  const int64_t s = t / strip, r = t - s * strip;
  const int64_t h = ta - s * 8 < 8 ? ta - s * 8 : 8;
  *a = s * 8 + r % h;
  *b = r / h;
}

// Second best and position of the best in one float: the value rounded away from zero far enough (towards +inf) that the
// low 7 bits are free.  Read as a float it is never below the value and at most 2^-15 of it above.
__device__ __forceinline__ float pack_second(float second, int pos) {
  u32 u = __float_as_uint(second);
  if (u >> 31) u = u > 0x800000FFu ? (u & ~0x7Fu) - 0x80u : 0u;
  else u = (u + 0x7Fu) & ~0x7Fu;
  return __uint_as_float(u | (u32)pos);
}

struct Best { float m, second; int pos; };
__device__ __forceinline__ Best join_best(Best a, Best b) {   // rows of a come before rows of b
  Best o;
  o.second = fmaxf(fminf(a.m, b.m), fmaxf(a.second, b.second));
  o.pos = b.m > a.m ? b.pos : a.pos;
  o.m = fmaxf(a.m, b.m);
  return o;
}
// of lanes whose rows interleave: the smaller position among equal maxima
__device__ __forceinline__ Best join_mixed(Best a, Best b) {
  Best o;
  o.second = fmaxf(fminf(a.m, b.m), fmaxf(a.second, b.second));
  o.pos = b.m > a.m ? b.pos : (a.m > b.m ? a.pos : (a.pos < b.pos ? a.pos : b.pos));
  o.m = fmaxf(a.m, b.m);
  return o;
}

// A component of a vector of any type
__device__ __forceinline__ float raw_component(const void* p, int64_t i, int dtype) {
  if (dtype == VS_FP32) return static_cast<const float*>(p)[i];
  if (dtype == VS_FP16) return (float)static_cast<const _Float16*>(p)[i];
  return (float)static_cast<const __bf16*>(p)[i];
}
// The components of vector a (the same in all lanes) that are infinite or NaN, times those of vector b (a lane's own): what the
// product of the two comes to, if b is finite elsewhere.
__device__ __forceinline__ float infinite_dot(const void* pa, int64_t a, const void* pb, int64_t b, int d, int dtype) {
  const int lane = lane_id();
  float s = 0.f;
  for (int k0 = 0; k0 < d; k0 += 64) {
    const float v = k0 + lane < d ? raw_component(pa, a * d + k0 + lane, dtype) : 0.f;
    for (u64 m = __ballot(!(fabsf(v) < __builtin_inff())); m; m &= m - 1) {
      const int t = __ffsll(m) - 1;
      s = __builtin_fmaf(__shfl(v, t), raw_component(pb, b * d + k0 + t, dtype), s);
      if (__ballot(s == s) == 0) return s;                  // (NaN for all)
    }
  }
  return s;
}

// The products of rows and queries with an infinite component, once more from the vectors: a head and a tail cannot hold an
// infinity (its product with a tail of the other side has any sign).  All of them are infinite or NaN, which the infinite
// factors of these rows and queries leave so.  A row, then a query at a time; a wavefront without either does not come here.
// row_bits: which of its rows, 64 to a word.
template <int IB, int JB>
__device__ __forceinline__ void infinite_products(const SmScores& S, int64_t a0, int64_t b0, const float2* rowdata,
                                                const u64* row_bits, f32x16 (&acc)[IB][JB]) {
  const int lane = lane_id(), wave = wave_id(), half = lane >> 5;
  const float2* mine = rowdata + (wave & 1) * 32 * IB;
  a0 += (wave & 1) * 32 * IB;
  b0 += (wave >> 1) * 32 * JB;
  const int64_t lane_q = b0 + lane % (32 * JB) < S.nq ? b0 + lane % (32 * JB) : S.nq - 1;
#pragma unroll 1
  for (int h = 0; h < IB / 2; ++h) {
    for (u64 m = row_bits[(wave & 1) * (IB / 2) + h]; m; m &= m - 1) {
      const int i = h * 64 + __ffsll(m) - 1;
      const float v = infinite_dot(S.raw_x, a0 + i, S.raw_q, lane_q, S.d, S.dtype);
      float s[JB];
#pragma unroll
      for (int jb = 0; jb < JB; ++jb) s[jb] = __shfl(v, jb * 32 + (lane & 31));
      const int at = i - 4 * half;
#pragma unroll
      for (int ib = 0; ib < IB; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
#pragma unroll
          for (int jb = 0; jb < JB; ++jb) acc[ib][jb][r] = at == ib * 32 + (r & 3) + 8 * (r >> 2) ? s[jb] : acc[ib][jb][r];
          __builtin_amdgcn_sched_barrier(0);                 // (a mask at a time: 64 of them leave no scalar register)
        }
    }
  }
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int64_t qi = b0 + jb * 32 + (lane & 31);
    for (u64 m = __ballot(lane < 32 && qi < S.nq && S.q.scale[qi < S.nq ? qi : 0] == __builtin_inff()); m; m &= m - 1) {
      const int c = __ffsll(m) - 1;
      float v[IB / 2];
#pragma unroll
      for (int h = 0; h < IB / 2; ++h) {
        const int64_t j = a0 + h * 64 + lane;
        v[h] = infinite_dot(S.raw_q, b0 + jb * 32 + c, S.raw_x, j < S.nx ? j : S.nx - 1, S.d, S.dtype);
      }
#pragma unroll
      for (int ib = 0; ib < IB; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int i = ib * 32 + (r & 3) + 8 * (r >> 2) + 4 * half;
          const float s = __shfl(v[ib / 2], i & 63) + (mine[i].x == __builtin_inff() ? acc[ib][jb][r] : 0.f);   // (both: both count)
          if ((lane & 31) == c) acc[ib][jb][r] = s;
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  }
}

// The scores of a wavefront's tile in place of its products: s = acc * (row factor * query factor) + bias, -inf for
// rows that do not exist (past the end, or bias -inf: whatever their products are).
// rowdata: LDS, {row factor, bias} of the workgroup's rows, filled here.
template <int IB, int JB>
__device__ __forceinline__ void finish_scores(const SmScores& S, int64_t a0, int64_t b0, float2* rowdata, f32x16 (&acc)[IB][JB]) {
  const int lane = lane_id(), wave = wave_id(), wa = wave & 1, wb = wave >> 1;
  const bool plain = S.x.scale == nullptr && S.bias == nullptr && a0 + 64 * IB <= S.nx;   // (the same in the workgroup)
  u64* row_bits = reinterpret_cast<u64*>(rowdata + 64 * IB);             // [IB] rows with an infinity that take part
  float cq[JB];
  bool odd = false;                                                      // (queries likewise)
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int64_t qi = b0 + (wb * JB + jb) * 32 + (lane & 31);
    cq[jb] = S.q.scale && qi < S.nq ? S.q.scale[qi] * 0x1p14f : 1.f;
    odd = odd || cq[jb] == __builtin_inff();
    cq[jb] *= S.scale;
  }
  u64 any = __ballot(odd);
  if (!plain) {
    const int64_t j = a0 + threadIdx.x;
    if (threadIdx.x < 64 * IB) {
      float xs = 1.f, b = neg_inf();
      if (j < S.nx) {
        if (S.x.scale) xs = S.x.scale[j] * 0x1p-14f;           // (prepared queries are up to 2^15: 2^14 goes over to their factor)
        b = S.bias ? S.bias[j] : 0.f;
      }
      rowdata[threadIdx.x] = make_float2(xs, b);
      const u64 bits = __ballot(b != neg_inf() && xs == __builtin_inff());
      if (lane == 0) row_bits[wave] = bits;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < IB / 2; ++h) any |= row_bits[wa * (IB / 2) + h];
    // (ahead of the scores, which are computed and used in one block of instructions)
    if (__builtin_expect(S.raw_x && __ballot(any != 0) != 0, 0)) infinite_products(S, a0, b0, rowdata, row_bits, acc);
  }
#pragma unroll
  for (int ib = 0; ib < IB; ++ib)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (plain) {
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) acc[ib][jb][r] *= cq[jb];
      } else {
        const float2 rd = rowdata[(wa * IB + ib) * 32 + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5)];
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) {
          const float s = acc[ib][jb][r] * rd.x * cq[jb] + rd.y;
          acc[ib][jb][r] = rd.y == neg_inf() ? neg_inf() : s;
        }
      }
    }
}

// ---- forward: scores -> softmax records ---------------------------------------------
// Bound by the matrix cores for long vectors and by the epilogue's exponentials (some 12 vector instructions per score)
// for short ones: bf16 4096 x 65,536 x 768 445 to 520 us with the clock, 790 to 930 TFLOP/s (the library's product of these
// sizes, stored, runs at 976); fp32 1000 x 200,003 x 100 in three products 242 to 251 us.  A wavefront's 128 rows are a record of
// each of its 64 queries.
template <int PLANES, bool BF16, bool SECOND>
__global__ __launch_bounds__(256, 2) void sm_scores_kernel(SmScores S, SmRecords R, int64_t ta, int64_t tb) {
  extern __shared__ __align__(16) char lds[];
  int64_t ia, ib_;
  tile_of(blockIdx.x, ta, tb, &ia, &ib_);
  const int64_t a0 = ia * kTileA, b0 = ib_ * kTileB;
  f32x16 acc[4][2] = {};
  TileMul<PLANES, BF16>::run(S.x, a0, S.q, b0, 0, S.kunits, lds, acc);
  finish_scores(S, a0, b0, reinterpret_cast<float2*>(lds), acc);
  const int lane = lane_id(), wave = wave_id(), wa = wave & 1, wb = wave >> 1, half = lane >> 5;
#pragma unroll
  for (int jb = 0; jb < 2; ++jb) {
    const int64_t qi = b0 + wb * 64 + jb * 32 + (lane & 31);
    float m = neg_inf(), second = neg_inf();
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float s = acc[ib][jb][r];
        if (SECOND) second = __builtin_amdgcn_fmed3f(s, m, second);
        m = fmaxf(m, s);
      }
    float w = 0.f;
    if (SECOND) {
      int pos = 0;
#pragma unroll
      for (int ib = 3; ib >= 0; --ib)
#pragma unroll
        for (int r = 15; r >= 0; --r)
          pos = acc[ib][jb][r] == m ? ib * 32 + (r & 3) + 8 * (r >> 2) + 4 * half : pos;
      const Best b = join_mixed(Best{m, second, pos}, Best{__shfl_xor(m, 32), __shfl_xor(second, 32), __shfl_xor(pos, 32)});
      m = b.m;
      w = pack_second(b.second, b.pos);
    } else {
      m = fmaxf(m, __shfl_xor(m, 32));
    }
    float l = 0.f, h = 0.f;
    const float base = m > neg_inf() ? m : 0.f;
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) softmax_add(acc[ib][jb][r] - base, &l, &h);
    l += __shfl_xor(l, 32);
    h += __shfl_xor(h, 32);
    if (R.keep && qi < S.nq)
#pragma unroll
      for (int ib = 0; ib < 4; ++ib)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int64_t j = a0 + wa * 128 + ib * 32 + 2 * r + 4 * half;   // keep_ld covers whole tiles: no tail
          *reinterpret_cast<float4*>(R.keep + qi * R.keep_ld + j) =
              make_float4(acc[ib][jb][r], acc[ib][jb][r + 1], acc[ib][jb][r + 2], acc[ib][jb][r + 3]);
        }
    const int64_t part = ia * 2 + wa;
    if (half == 0 && qi < S.nq && part < R.parts) R.rec[qi * R.parts + part] = make_float4(m, l, h, w);
  }
}

// ---- forward for few queries ----------------------------------------------------------
// Up to 64 queries the rows are what there is to read: a wavefront loads fragments of 32 rows straight from memory
// (no LDS, 16 bytes a lane and load) and multiplies them with all queries, whose fragments wait in LDS; four wavefronts
// make the record of 128 rows.  fp32 rows use v_mfma_f32_16x16x4_f32: exact products, and its 157 TFLOP/s are far above
// what the stream of rows can ask for.  Bound by memory: bf16 100,003 x 768, one query, 33.3 us, 4.6 TB/s for a copy's 4.7.
// In the 16x16 layouts a lane holds row lane & 15 of A, and of the result column lane & 15 and rows 4 (lane >> 4) + r.
template <int DT>
struct FewMul {
  typedef typename Elem<DT>::T T;
  static constexpr int KS = DT == 0 ? 16 : 32;        // K elements per step: 16 bytes for each of 4 lane groups
  static constexpr int PER = DT == 0 ? 4 : 8;         // of them in a lane
  static __device__ __forceinline__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (DT == 0) {
      const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
      return c;
    } else if constexpr (DT == 1) {
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
  }
  // PER elements k .. of a row of d, zeros past its end
  static __device__ __forceinline__ u32x4 load(const T* row, int k, int d) {
    u32x4 v;
    if (k + PER <= d) {
      __builtin_memcpy(&v, row + k, 16);
    } else {
      T e[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) e[i] = k + i < d ? row[k + i] : (T)0.f;
      __builtin_memcpy(&v, e, 16);
    }
    return v;
  }
};

constexpr int kFewChunkBytes = 64 * 1024;             // of query fragments in LDS
template <int DT, int NT>
constexpr int few_chunk() { return kFewChunkBytes / (NT * 1024) * FewMul<DT>::KS; }   // K elements of a chunk

template <int DT, int NT, bool SECOND>
__global__ __launch_bounds__(256) void sm_scores_few_kernel(const typename Elem<DT>::T* __restrict__ x, int64_t nb,
                                                            const typename Elem<DT>::T* __restrict__ q, int nq, int d,
                                                            float scale, const float* __restrict__ bias, SmRecords R) {
  typedef FewMul<DT> F;
  constexpr int CH = few_chunk<DT, NT>();
  extern __shared__ __align__(16) char lds[];
  u32x4* frag = reinterpret_cast<u32x4*>(lds);        // [step][NT][64]
  const int lane = lane_id(), wave = wave_id(), g = lane >> 4;
  const int64_t part = group_id(), j0 = part * kSmRecRows + wave * 32;
  if (part >= R.parts) return;
  const typename F::T* row[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int64_t j = j0 + i * 16 + (lane & 15);
    row[i] = x + (j < nb ? j : nb - 1) * d;
  }
  f32x4 acc[2][NT] = {};
  for (int c0 = 0; c0 < d; c0 += CH) {
    const int c1 = c0 + CH < d ? c0 + CH : d, steps = (c1 - c0 + F::KS - 1) / F::KS;
    if (c0 > 0) __syncthreads();
    for (int i = threadIdx.x; i < steps * NT * 64; i += 256) {
      const int l = i & 63, t = (i >> 6) % NT, s = (i >> 6) / NT, qi = t * 16 + (l & 15);
      u32x4 v = {0, 0, 0, 0};
      if (qi < nq) v = F::load(q + (int64_t)qi * d, c0 + s * F::KS + (l >> 4) * F::PER, d);
      frag[i] = v;
    }
    __syncthreads();
    constexpr int U = 8;
    int s = 0;
    for (; s + U <= steps && c0 + (s + U) * F::KS <= d; s += U) {
      u32x4 a[U][2];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) __builtin_memcpy(&a[u][i], row[i] + c0 + (s + u) * F::KS + g * F::PER, 16);
      __builtin_amdgcn_sched_barrier(0);              // (all sixteen loads leave before the first is waited for)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const u32x4 b = frag[((s + u) * NT + t) * 64 + lane];
          acc[0][t] = F::mul(a[u][0], b, acc[0][t]);
          acc[1][t] = F::mul(a[u][1], b, acc[1][t]);
        }
      settle_products();
    }
    for (; s < steps; ++s) {
      const int k = c0 + s * F::KS + g * F::PER;
      const u32x4 a0 = F::load(row[0], k, d), a1 = F::load(row[1], k, d);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const u32x4 b = frag[(s * NT + t) * 64 + lane];
        acc[0][t] = F::mul(a0, b, acc[0][t]);
        acc[1][t] = F::mul(a1, b, acc[1][t]);
      }
      settle_products();
    }
  }
  __syncthreads();
  float4* recs = reinterpret_cast<float4*>(lds);                   // [4][NT * 16]
  float* seconds = reinterpret_cast<float*>(lds + 4 * NT * 16 * 16);
  float bj[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t j = j0 + i * 16 + 4 * g + r;
      bj[i][r] = j < nb ? (bias ? bias[j] : 0.f) : neg_inf();
    }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float m = neg_inf(), second = neg_inf();
    float s[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float v = acc[i][t][r] * scale + bj[i][r];
        s[i][r] = bj[i][r] == neg_inf() ? neg_inf() : v;
        if (SECOND) second = __builtin_amdgcn_fmed3f(s[i][r], m, second);
        m = fmaxf(m, s[i][r]);
      }
    const int qi = t * 16 + (lane & 15);
    if (R.keep && qi < nq)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<float4*>(R.keep + (int64_t)qi * R.keep_ld + j0 + i * 16 + 4 * g) =
            make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
    Best b{m, second, 0};
    if (SECOND) {
#pragma unroll
      for (int i = 1; i >= 0; --i)
#pragma unroll
        for (int r = 3; r >= 0; --r) b.pos = s[i][r] == m ? wave * 32 + i * 16 + 4 * g + r : b.pos;
    }
#pragma unroll
    for (int w = 16; w <= 32; w <<= 1) {
      if (SECOND) b = join_mixed(b, Best{__shfl_xor(b.m, w), __shfl_xor(b.second, w), __shfl_xor(b.pos, w)});
      else b.m = fmaxf(b.m, __shfl_xor(b.m, w));
    }
    float l = 0.f, h = 0.f;
    const float base = b.m > neg_inf() ? b.m : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) softmax_add(s[i][r] - base, &l, &h);
#pragma unroll
    for (int w = 16; w <= 32; w <<= 1) { l += __shfl_xor(l, w); h += __shfl_xor(h, w); }
    if (g == 0) {
      recs[wave * NT * 16 + qi] = make_float4(b.m, l, h, __int_as_float(b.pos));
      seconds[wave * NT * 16 + qi] = b.second;
    }
  }
  __syncthreads();
  const int qi = threadIdx.x;
  if (qi >= nq || qi >= NT * 16) return;
  Best b{neg_inf(), neg_inf(), 0};
  for (int w = 0; w < 4; ++w) {
    const float4 o = recs[w * NT * 16 + qi];
    b = join_best(b, Best{o.x, seconds[w * NT * 16 + qi], __float_as_int(o.w)});
  }
  float l = 0.f, h = 0.f;
  for (int w = 0; w < 4; ++w) {
    const float4 o = recs[w * NT * 16 + qi];
    softmax_join(b.m, o.x, o.y, o.z, &l, &h);
  }
  R.rec[(int64_t)qi * R.parts + part] = make_float4(b.m, l, h, SECOND ? pack_second(b.second, b.pos) : 0.f);
}

// ---- finish: records -> normaliser, entropy, targets, alternatives ------------------------
// <q, x_j> for eight rows at once, eight lanes a row; every lane of a row's group gets the sum.  LANES = 64: one row.
template <int LANES, typename T>
__device__ __forceinline__ float dot_rows(const T* __restrict__ q, const T* __restrict__ row, int d) {
  constexpr int V = 16 / sizeof(T);
  const int l = lane_id() & (LANES - 1);
  float acc = 0.f;
  int k = l * V;
#pragma unroll 4
  for (; k + V <= d; k += LANES * V) {
    T a[V], b[V];
    __builtin_memcpy(a, q + k, 16);
    __builtin_memcpy(b, row + k, 16);
#pragma unroll
    for (int i = 0; i < V; ++i) acc = __builtin_fmaf(to_f32(a[i]), to_f32(b[i]), acc);
  }
  for (int i = k; i < d && i < k + V; ++i) acc = __builtin_fmaf(to_f32(q[i]), to_f32(row[i]), acc);
#pragma unroll
  for (int w = 1; w < LANES; w <<= 1) acc += __shfl_xor(acc, w);
  return acc;
}

// Maximum over the wavefront in every lane: inside rows of 16 lanes by DPP, across them by two broadcasts.
__device__ __forceinline__ float wave_max_dpp(float v) {
  auto step = [&](int o) { v = fmaxf(v, __int_as_float(o)); };
  const int lo = __float_as_int(neg_inf());
  step(__builtin_amdgcn_update_dpp(lo, __float_as_int(v), 0x111, 0xF, 0xF, false));   // row_shr 1, 2, 4, 8
  step(__builtin_amdgcn_update_dpp(lo, __float_as_int(v), 0x112, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(lo, __float_as_int(v), 0x114, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(lo, __float_as_int(v), 0x118, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(lo, __float_as_int(v), 0x142, 0xA, 0xF, false));   // row_bcast 15, 31
  step(__builtin_amdgcn_update_dpp(lo, __float_as_int(v), 0x143, 0xC, 0xF, false));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// A score as what it is ordered by: keys tell zeros of different signs apart, which are equal scores (a negative scale, a
// scale of zero and a bias of -0 make such).
__device__ __forceinline__ float rank_value(float s) { return s + 0.f; }

constexpr int kTakeBest = 16, kTakePer = 8;
// The k best of the wavefront's records (thread's i-th: threadIdx.x + 256 i) as ascending keys of {maximum, record}: the
// best of the lanes' bests k times, its lane going through its own again.
__device__ __forceinline__ void wave_take_best(const float4 (&rec)[kTakePer], int k, u64* out) {
  u32 gone = 0;                                           // which of this lane's are taken
  float best;
  int at;
  auto mine = [&]() {
    best = neg_inf();
    at = 0;
#pragma unroll
    for (int i = 0; i < kTakePer; ++i)
      if (rec[i].x > best && !((gone >> i) & 1u)) { best = rec[i].x; at = i; }
  };
  mine();
  for (int r = 0; r < k; ++r) {
    const float top = wave_max_dpp(best);
    u64 key = KEY_EMPTY;
    if (top > neg_inf()) {
      const u32 id = threadIdx.x + 256u * (u32)at;
      u64 have = __ballot(best == top);
      u32 win = __builtin_amdgcn_readlane((int)id, __ffsll(have) - 1);
      for (have &= have - 1; have; have &= have - 1) {    // equal maxima: the smaller record
        const u32 o = __builtin_amdgcn_readlane((int)id, __ffsll(have) - 1);
        win = o < win ? o : win;
      }
      key = make_key(top, win, 1);
      if (best == top && id == win) { gone |= 1u << at; mine(); }
    }
    if (lane_id() == 0) out[r] = key;
  }
}

// One workgroup per query.  The k best rows lie in the k records with the best maxima (a row outside them is beaten by k
// maxima; records cover consecutive rows, so ties fall to the smaller row as well).  Of such a record only the maximum
// can count unless its second best reaches the k-th best maximum: then its 128 scores are computed again in fp32.
// Where that would be common (few records, or many alternatives) the scores have been kept, and are read instead.
// TAKE: up to kTakeBest alternatives of up to 256 kTakePer records (262,144 rows), which stay in registers and are picked
// one by one; more go through the reservoir selection, whose first sort alone takes some 700 instructions.  A chain of
// latencies: one query of 782 records, k = 10, 12.1 us; 4096 queries of 512 records, k = 5, 62 us.
template <int DT, bool TAKE>
__global__ __launch_bounds__(256) void sm_finish_kernel(SmFinish F, SmRecords R) {
  typedef typename Elem<DT>::T T;
  constexpr int TOT = 128;
  __shared__ u64 slots[4 * TOT];
  __shared__ u64 chosen[VS_MAX_TOP];
  __shared__ u64 shared_bound;
  __shared__ float red[3][4];
  const int64_t qi = group_id();
  if (qi >= F.nq) return;
  const int lane = lane_id(), wave = wave_id();
  const float4* rec = R.rec + qi * R.parts;
  const T* x = static_cast<const T*>(F.x);
  const T* q = static_cast<const T*>(F.q) + qi * F.d;
  const int64_t target = wave < F.nt ? F.targets[qi * F.nt + wave] : -1;
  const bool target_in = target >= 0 && target < F.nb;
  float m = neg_inf();
  float4 own[TAKE ? kTakePer : 1];
  if (TAKE) {
#pragma unroll
    for (int i = 0; i < kTakePer; ++i) {
      const int64_t p = threadIdx.x + 256 * i;
      own[i] = p < R.parts ? rec[p] : make_float4(neg_inf(), 0.f, 0.f, 0.f);
      own[i].x = rank_value(own[i].x);
    }
#pragma unroll
    for (int i = 0; i < kTakePer; ++i) m = fmaxf(m, own[i].x);
  } else {
#pragma unroll 4
    for (int64_t p = threadIdx.x; p < R.parts; p += 256) m = fmaxf(m, rec[p].x);
  }
  // (of target `wave`, while the records are on their way)
  const float target_score = wave < F.nt && F.nb > 0 ? dot_rows<64>(q, x + (target_in ? target : 0) * F.d, F.d) : 0.f;
  m = wave_max_dpp(m);
  if (lane == 0) red[0][wave] = m;
  if (threadIdx.x == 0) shared_bound = KEY_EMPTY;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  float l = 0.f, h = 0.f;
  if (TAKE) {
#pragma unroll
    for (int i = 0; i < kTakePer; ++i) softmax_join(m, own[i].x, own[i].y, own[i].z, &l, &h);
  } else {
#pragma unroll 4
    for (int64_t p = threadIdx.x; p < R.parts; p += 256) {
      const float4 r = rec[p];
      softmax_join(m, r.x, r.y, r.z, &l, &h);
    }
  }
  l = wave_sum(l);
  h = wave_sum(h);
  if (lane == 0) { red[1][wave] = l; red[2][wave] = h; }
  if constexpr (TAKE) {
    if (F.k > 0) wave_take_best(own, F.k, slots + wave * TOT);
  }
  __syncthreads();
  l = red[1][0] + red[1][1] + red[1][2] + red[1][3];
  h = red[2][0] + red[2][1] + red[2][2] + red[2][3];
  const bool empty = m == neg_inf() && l == 0.f;
  const float logl = empty ? 0.f : logf(l), lse = empty ? neg_inf() : m + logl;
  if (threadIdx.x == 0) {
    F.lse[qi] = lse;
    F.entropy[qi] = empty ? 0.f : logl - h / l;
  }
  for (int t = wave; t < F.nt; t += 4) {
    const int64_t j = t < 4 ? target : F.targets[qi * F.nt + t];
    const bool in = j >= 0 && j < F.nb;
    const float b = in && F.bias ? F.bias[j] : 0.f;
    const float dot = t < 4 || F.nb == 0 ? target_score : dot_rows<64>(q, x + (in ? j : 0) * F.d, F.d);
    if (lane == 0) F.logp[qi * F.nt + t] = !in ? 0.f : (b == neg_inf() ? neg_inf() : dot * F.scale + b - lse);
  }
  if (F.k == 0) return;
  WaveSelect<2> sel;
  auto start = [&]() {
    sel.init(slots + wave * TOT, TOT, F.k, &shared_bound);
    sel.set_metric(1);
  };
  const KeySink to{chosen, nullptr, nullptr, nullptr, nullptr, 1};
  const int group = lane >> 3;
  bool done = false;
  if (R.keep) {
    start();
    const float* s = R.keep + qi * R.keep_ld;
    for (int64_t j0 = wave * 64; j0 < F.nb; j0 += 256) {
      const int64_t j = j0 + lane;
      const float v = j < F.nb ? rank_value(s[j]) : neg_inf();
      sel.push_value(v > neg_inf(), v, (u32)j);
    }
  } else {
    if (!TAKE) {
      start();
      for (int64_t p0 = wave * 64; p0 < R.parts; p0 += 256) {
        const int64_t p = p0 + lane;
        const float v = p < R.parts ? rank_value(rec[p].x) : neg_inf();
        sel.push_value(v > neg_inf(), v, (u32)p);
      }
      sel.finish();
      __syncthreads();
    }
    if (TAKE) {                                             // 4 k <= 64 keys, one a lane, to their places
      if (wave == 0) {
        const u64 mine = lane < 4 * F.k ? slots[lane / F.k * TOT + lane % F.k] : KEY_EMPTY;
        int rank = 0;
        for (int i = 0; i < 4 * F.k; ++i) {
          const u64 o = __shfl(mine, i);
          rank += o < mine || (o == mine && i < lane) ? 1 : 0;
        }
        if (lane < 4 * F.k && rank < F.k) chosen[rank] = mine;
      }
    } else {
      block_rank_merge(slots, TOT, 4, F.k, to, 0);
    }
    if (threadIdx.x == 0) shared_bound = KEY_EMPTY;
    __syncthreads();
    // (VS_MAX_TOP = 64: one lane holds each of the chosen records)
    const u64 last = chosen[F.k - 1], key = lane < F.k ? chosen[lane] : KEY_EMPTY;
    const float tau = last == KEY_EMPTY ? neg_inf() : key_value(last, 1);
    const u32 p = key_index(key);
    const float w = key != KEY_EMPTY ? rec[p].w : 0.f;
    const bool whole = key != KEY_EMPTY && w >= tau;
    const u32 lone_row = p * kSmRecRows + (__float_as_uint(w) & 127u);
    const u64 todo = __ballot(whole);
    __syncthreads();                                        // (everybody has read what was chosen)
    if (todo == 0) {                                        // the maxima are the best rows, in this order
      if (wave == 0 && lane < F.k) chosen[lane] = key == KEY_EMPTY ? KEY_EMPTY : make_key(key_value(key, 1), lone_row, 1);
      done = true;
    } else {
      // the maxima that stand alone, then whole records, 32 rows a step (all of them: equal rows must meet with equal bits)
      start();
      const u64 lone = __ballot(key != KEY_EMPTY && !whole);
      const int lones = (F.k + 31) / 32, steps = lones + 4 * __popcll(todo);
      u64 rest = todo;
      u32 pw = 0;
      for (int t = 0; t < steps; ++t) {
        const int i = wave * 8 + group;                     // of the step's rows
        int64_t j;
        bool in = true;
        if (t < lones) {
          j = __shfl(lone_row, t * 32 + i);
          in = (lone >> (t * 32 + i)) & 1u;
        } else {
          const int r = (t - lones) & 3;
          if (r == 0) { pw = __shfl(p, __ffsll(rest) - 1); rest &= rest - 1; }
          j = (int64_t)pw * kSmRecRows + r * 32 + i;
        }
        in = in && j < F.nb;
        const float b = in ? (F.bias ? F.bias[j] : 0.f) : neg_inf();
        const float s = rank_value(dot_rows<8>(q, x + (in ? j : 0) * F.d, F.d) * F.scale + b);
        sel.push_value((lane & 7) == 0 && b > neg_inf() && s > neg_inf(), s, (u32)j);
      }
    }
  }
  if (!done) {
    sel.finish();
    __syncthreads();
    block_rank_merge(slots, TOT, 4, F.k, to, 0);
  }
  __syncthreads();
  if ((int)threadIdx.x < F.k) {
    const u64 key = chosen[threadIdx.x];
    F.top_logp[qi * F.k + threadIdx.x] = key == KEY_EMPTY ? neg_inf() : key_value(key, 1) - lse;
    F.top_ids[qi * F.k + threadIdx.x] = key == KEY_EMPTY ? -1 : (int64_t)key_index(key);
  }
}

// ---- preparation of operands ------------------------------------------------------------
__device__ __forceinline__ void row_scale(float mx, float* up, float* down) {
  const int e = top_exponent(mx);
  *up = __builtin_ldexpf(1.f, e);
  *down = __builtin_ldexpf(1.f, -e);
}
// Elements k .. k + 15 / sizeof(T) of a row as floats, zeros past its end (one load wherever the row begins)
template <typename T>
__device__ __forceinline__ void load_piece(const T* __restrict__ row, int k, int d, float (&v)[16 / sizeof(T)]) {
  constexpr int V = 16 / sizeof(T);
  if (k + V <= d) {
    T e[V];
    __builtin_memcpy(e, row + k, 16);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = to_f32(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = k + i < d ? to_f32(row[k + i]) : 0.f;
  }
}

// 16 lanes a row, 16 bytes a lane and step; rows of up to kPrepSteps steps are read once and stay in registers.  Bound by
// memory: 201,003 x 100 fp32 into two planes 30 us, 183 MB at 6.1 TB/s (part of it stays in the last-level cache).
constexpr int kPrepSteps = 8;
template <int DT, int PLANES>
__global__ __launch_bounds__(256) void sm_prep_rows_kernel(SmSide side0, SmSide side1, unsigned blocks0, int d, int64_t dp) {
  typedef typename Elem<DT>::T T;
  constexpr int V = 16 / sizeof(T);
  const int64_t wg = group_id();
  const SmSide& S = wg < blocks0 ? side0 : side1;
  const T* __restrict__ x = static_cast<const T*>(S.x);
  const float* __restrict__ bias = S.bias;
  char* __restrict__ planes = static_cast<char*>(S.rows);
  float* __restrict__ scale = S.row_scale;
  const int64_t r = (wg < blocks0 ? wg : wg - blocks0) * 16 + (threadIdx.x >> 4);
  if (r >= S.n) return;                                                // (whole groups of 16 lanes)
  const int l = threadIdx.x & 15;
  const bool gone = bias && bias[r] == neg_inf(), kept = dp <= 16 * V * kPrepSteps;
  const T* row = x + r * d;
  float v[kPrepSteps][V];
  u32 mx = 0;                                                          // the largest size, as bits: a NaN is above infinity
  auto take = [&](float e) {
    const u32 b = __float_as_uint(e) & 0x7FFFFFFFu;
    mx = b > mx ? b : mx;
  };
  if (kept) {
#pragma unroll
    for (int i = 0; i < kPrepSteps; ++i) {
      const int k = (i * 16 + l) * V;
#pragma unroll
      for (int u = 0; u < V; ++u) v[i][u] = 0.f;
      if (!gone && k < d) load_piece(row, k, d, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kPrepSteps; ++i)
#pragma unroll
      for (int u = 0; u < V; ++u) take(v[i][u]);
  } else if (!gone) {
    for (int k = l * V; k < d; k += 16 * V) {
      load_piece(row, k, d, v[0]);
#pragma unroll
      for (int u = 0; u < V; ++u) take(v[0][u]);
    }
  }
#pragma unroll
  for (int w = 1; w < 16; w <<= 1) take(__uint_as_float(__shfl_xor(mx, w)));
  float up, down;
  row_scale(__uint_as_float(mx), &up, &down);
  char* out = planes + r * (dp * 2 * PLANES);
  auto put = [&](int64_t k, const float (&e)[V]) {
    _Float16 hi[V], lo[V];
#pragma unroll
    for (int u = 0; u < V; ++u) {
      const float t = e[u] * up;
      hi[u] = (_Float16)t;
      lo[u] = (_Float16)(t - (float)hi[u]);
    }
    char* to = PLANES == 1 ? out + k * 2 : out + (k >> 4) * 64 + (k & 15) * 2;
    __builtin_memcpy(to, hi, sizeof(hi));
    if (PLANES == 2) __builtin_memcpy(to + 32, lo, sizeof(lo));
  };
  if (kept) {
#pragma unroll
    for (int i = 0; i < kPrepSteps; ++i) {
      const int64_t k = (i * 16 + l) * V;
      if (k < dp) put(k, v[i]);
    }
  } else {
    for (int64_t k = l * V; k < dp; k += 16 * V) {
#pragma unroll
      for (int u = 0; u < V; ++u) v[0][u] = 0.f;
      if (!gone && k < d) load_piece(row, (int)k, d, v[0]);
      put(k, v[0]);
    }
  }
  // (a NaN makes the row's scores NaN, an infinity leaves them to infinite_products)
  if (l == 0) scale[r] = mx < 0x7F800000u ? down : __uint_as_float(mx);
}

// Largest size in every column: a thread goes down 16 bytes of columns, four rows in flight, as many rows beside each
// other as a wavefront holds.  (A maximum does not depend on the order, and non-negative floats are ordered as their
// bits.)  Bound by memory where rows are long: 69,632 x 768 bf16 39 us, 2.7 TB/s; 30,788 x 100 fp16 15 us.
template <int DT>
__global__ __launch_bounds__(256) void sm_colmax_kernel(SmSide side0, SmSide side1, unsigned blocks0, int d, int64_t rows_per) {
  typedef typename Elem<DT>::T T;
  constexpr int V = 16 / sizeof(T);
  const SmSide& S = blockIdx.y < blocks0 ? side0 : side1;
  const T* __restrict__ x = static_cast<const T*>(S.x);
  const float* __restrict__ bias = S.bias;
  const float* __restrict__ factor = S.factor;
  u32* __restrict__ colmax = S.colmax;
  const int64_t n = S.n;
  __shared__ float part[4][64 * V];
  int row_lanes = 64;                                        // lanes that share a row: a power of two
  while (row_lanes > 1 && row_lanes / 2 * V >= d) row_lanes >>= 1;
  const int lane = lane_id(), wave = wave_id(), apart = 4 * (64 / row_lanes);
  // a lane's columns: the last ones of a row where V of them would end behind it (a column may be seen twice)
  auto columns = [&](int c) {
    const int t = (blockIdx.x * 64 + c) * V;
    return t >= d ? -1 : (t + V <= d ? t : (d > V ? d - V : 0));
  };
  const int t = columns(lane % row_lanes);
  const int64_t r0 = (int64_t)(blockIdx.y < blocks0 ? blockIdx.y : blockIdx.y - blocks0) * rows_per;
  const int64_t r1 = r0 + rows_per < n ? r0 + rows_per : n;
  float mx[V] = {};
  if (t >= 0)
    for (int64_t r = r0 + (wave * 64 + lane) / row_lanes; r < r1; r += 4 * apart) {
      int64_t row[4];                                        // (the last one again behind the end)
      float v[4][V], f[4] = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) row[i] = r + i * apart < r1 ? r + i * apart : r1 - 1;
      if (d >= V) {
        T e[4][V];
#pragma unroll
        for (int i = 0; i < 4; ++i) __builtin_memcpy(e[i], x + row[i] * d + t, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int u = 0; u < V; ++u) v[i][u] = to_f32(e[i][u]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) load_piece(x + row[i] * d, 0, d, v[i]);
      }
      if (factor)
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = factor[row[i]];
      if (bias) {
        float b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = bias[row[i]];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = b[i] == neg_inf() ? 0.f : f[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < V; ++u) mx[u] = f[i] != 0.f ? fmaxf(mx[u], fabsf(v[i][u]) * f[i]) : mx[u];
    }
  for (int w = row_lanes; w < 64; w <<= 1)
#pragma unroll
    for (int u = 0; u < V; ++u) mx[u] = fmaxf(mx[u], __shfl_xor(mx[u], w));
#pragma unroll
  for (int i = 0; i < V; ++i) part[wave][lane * V + i] = mx[i];
  __syncthreads();
  for (int i = threadIdx.x; i < row_lanes * V; i += 256) {
    const float m = fmaxf(fmaxf(part[0][i], part[1][i]), fmaxf(part[2][i], part[3][i]));
    const int c = columns(i / V);
    if (c >= 0 && c + i % V < d && m > 0.f) atomicMax(colmax + c + i % V, __float_as_uint(m));
  }
}

// 64 rows x 64 columns through LDS: column t becomes a row of K blocks over r, read and written in 16-byte pieces.
// 69,632 x 768 bf16: 65 us, 214 MB at 3.3 TB/s.
template <int DT, int PLANES>
__global__ __launch_bounds__(256) void sm_prep_cols_kernel(SmSide side0, SmSide side1, unsigned blocks0, int d) {
  typedef typename Elem<DT>::T T;
  constexpr int V = 16 / sizeof(T);
  __shared__ float tile[64][65];
  const int64_t wg = blockIdx.x + (int64_t)gridDim.x * blockIdx.z;
  const SmSide& S = wg < blocks0 ? side0 : side1;
  const T* __restrict__ x = static_cast<const T*>(S.x);
  const float* __restrict__ bias = S.bias;
  const float* __restrict__ factor = S.factor;
  const u32* __restrict__ colmax = S.colmax;
  char* __restrict__ planes = static_cast<char*>(S.cols);
  float* __restrict__ scale = S.col_scale;
  const int64_t n = S.n, np = S.np;
  const int64_t r0 = (wg < blocks0 ? wg : wg - blocks0) * 64;
  const int t0 = blockIdx.y * 64;
  for (int i = threadIdx.x; i < 64 * 64 / V; i += 256) {
    const int row = i / (64 / V), c = i % (64 / V) * V;
    const int64_t r = r0 + row;
    float v[V] = {};
    const float f = r < n && !(bias && bias[r] == neg_inf()) ? (factor ? factor[r] : 1.f) : 0.f;
    if (f != 0.f && t0 + c < d) load_piece(x + r * d, t0 + c, d, v);
#pragma unroll
    for (int u = 0; u < V; ++u) tile[row][c + u] = f != 0.f ? v[u] * f : 0.f;   // (what takes no part may be a NaN)
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * 8; i += 256) {
    const int c = i & 63, k = (i >> 6) * 8, t = t0 + c;
    if (t >= d || r0 + k >= np) continue;
    float up, down;
    row_scale(__uint_as_float(colmax[t]), &up, &down);
    f16x8 hi, lo;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float v = tile[k + u][c] * up;
      hi[u] = (_Float16)v;
      lo[u] = (_Float16)(v - (float)hi[u]);
    }
    char* out = planes + (int64_t)t * (np * 2 * PLANES);
    const int64_t kk = r0 + k;
    if (PLANES == 1) {
      *reinterpret_cast<f16x8*>(out + kk * 2) = hi;
    } else {
      *reinterpret_cast<f16x8*>(out + (kk >> 4) * 64 + (kk & 15) * 2) = hi;
      *reinterpret_cast<f16x8*>(out + (kk >> 4) * 64 + 32 + (kk & 15) * 2) = lo;
    }
    if (r0 == 0 && k == 0) scale[t] = down;
  }
}

// ---- backward ------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void sm_coefs_kernel(SmGrads g, int64_t nq, int64_t nb, float4* __restrict__ coef,
                                                       float* __restrict__ bound, u32* __restrict__ clear, int n_clear) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t c = i; c < n_clear; c += (int64_t)gridDim.x * 256) clear[c] = 0;
  if (i >= nq) return;
  float sum = 0.f, mag = 0.f;
  if (g.g_logp)
    for (int t = 0; t < g.nt; ++t) {
      const int64_t j = g.targets[i * g.nt + t];
      if (j < 0 || j >= nb) continue;
      const float v = g.g_logp[i * g.nt + t];
      sum += v;
      mag += fabsf(v);
    }
  const float c = (g.g_lse ? g.g_lse[i] : 0.f) - sum;
  const float ge = g.g_entropy ? g.g_entropy[i] : 0.f, ent = g.g_entropy ? g.entropy[i] : 0.f;
  // |G| <= |c| p + |g_entropy| (p |logp| + p H) + sum |g_logp|, and p |logp| <= 1 / e
  const float top = fabsf(c) + mag + fabsf(ge) * (0.37f + fabsf(ent));
  int e = top > 0.f && top < __builtin_inff() ? (int)__builtin_amdgcn_frexp_expf(top) : 0;
  e = e < -100 ? -100 : (e > 127 ? 127 : e);
  // 0, a padded query: it takes no part, whatever it holds.  Infinite or NaN: G is NaN for the rows that exist (an infinite
  // coefficient would leave infinities among them, and -inf marks a row that does not).
  const bool bad = !(top < __builtin_inff());
  bound[i] = top == 0.f || bad ? top : __builtin_ldexpf(1.f, e);
  coef[i] = make_float4(bad ? __builtin_nanf("") : c, ge, ent, top == 0.f ? neg_inf() : g.lse[i]);
}

// Scores again, then G in place of them, as operands of the two products that follow: G [nq][rows] and its transpose.
// G / bound 2^14 in fp16: a value keeps 11 bits (22 with a tail) down to 2^-28 of the bound and 2^-38 of it below.
// Bound by the matrix cores and the stores of G: bf16 4096 x 16,384 x 768 210 us, 490 TFLOP/s beside 268 MB at 1.3 TB/s.
template <int PLANES, bool BF16, int IB, int JB>
__global__ __launch_bounds__(256, 2) void sm_gradients_kernel(SmScores S, SmGOut O, int64_t ta, int64_t tb) {
  extern __shared__ __align__(16) char lds[];
  int64_t ia, ib_;
  tile_of(blockIdx.x, ta, tb, &ia, &ib_);
  constexpr int TA = 64 * IB, TB = 64 * JB;
  const int64_t a0 = ia * TA, b0 = ib_ * TB;
  f32x16 acc[IB][JB] = {};
  TileMul<PLANES, BF16, IB, JB>::run(S.x, a0, S.q, b0, 0, S.kunits, lds, acc);
  finish_scores(S, a0, b0, reinterpret_cast<float2*>(lds), acc);
  const int lane = lane_id(), wave = wave_id(), wa = wave & 1, wb = wave >> 1, half = lane >> 5;
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int64_t qi = b0 + (wb * JB + jb) * 32 + (lane & 31);
    const bool in = qi < S.nq;
    const float4 c = in ? O.coef[qi] : make_float4(0.f, 0.f, 0.f, neg_inf());
    const bool some = c.w != neg_inf();
#pragma unroll
    for (int ib = 0; ib < IB; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float s = acc[ib][jb][r];
        const float logp = s - c.w;
        const float v = exp_neg(logp) * (c.x - c.y * (fmaxf(logp, -1000.f) + c.z));
        // a row that does not exist carries the mark of its score until the targets are in
        acc[ib][jb][r] = s == neg_inf() || !some ? neg_inf() : v;
      }
    if (O.g_logp && in)
      for (int t = 0; t < O.nt; ++t) {
        const int64_t j = O.targets[qi * O.nt + t] - O.row0 - a0 - wa * 32 * IB;  // relative to the wavefront's rows
        if (j >= 0 && j < 32 * IB) {
          const float gl = O.g_logp[qi * O.nt + t];
#pragma unroll
          for (int ib = 0; ib < IB; ++ib)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if ((int)j == ib * 32 + (r & 3) + 8 * (r >> 2) + 4 * half) acc[ib][jb][r] += gl;
        }
      }
#pragma unroll
    for (int ib = 0; ib < IB; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[ib][jb][r] = acc[ib][jb][r] == neg_inf() ? 0.f : acc[ib][jb][r];
  }
  __syncthreads();                                                  // (rowdata has been read)
  if (O.db) {                                                       // column sums of this tile, in a fixed order
    float* dbs = reinterpret_cast<float*>(lds);                     // [2][TA]
#pragma unroll
    for (int ib = 0; ib < IB; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float v = acc[ib][0][r] + (JB == 2 ? acc[ib][JB - 1][r] : 0.f);
        v += __uint_as_float(lane_xor_u32<1>(__float_as_uint(v)));
        v += __uint_as_float(lane_xor_u32<2>(__float_as_uint(v)));
        v += __uint_as_float(lane_xor_u32<4>(__float_as_uint(v)));
        v += __uint_as_float(lane_xor_u32<8>(__float_as_uint(v)));
        v += __shfl_xor(v, 16);
        if ((lane & 31) == 0) dbs[wb * TA + (wa * IB + ib) * 32 + (r & 3) + 8 * (r >> 2) + 4 * half] = v;
      }
    __syncthreads();
    if (threadIdx.x < TA && a0 + threadIdx.x < S.nx)
      O.db[ib_ * O.db_ld + a0 + threadIdx.x] = dbs[threadIdx.x] + dbs[TA + threadIdx.x];
    __syncthreads();
  }
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int64_t qi = b0 + (wb * JB + jb) * 32 + (lane & 31);
    const float bnd = qi < S.nq ? O.bound[qi] : 0.f;
    const float inv = bnd == 0.f ? 0.f : 16384.f / bnd;
#pragma unroll
    for (int ib = 0; ib < IB; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[ib][jb][r] *= inv;
  }
  // Out through LDS, 128 rows at a time: the wavefronts that hold them write, all copy.
  constexpr int LDG = 2 * 128 + 16, LDT = 2 * TB + 16;              // bytes of a row of the staged tiles
  constexpr int PER = PLANES == 2 ? 16 : 32;                        // elements of a K unit
  for (int plane = 0; plane < PLANES; ++plane) {
    for (int h = 0; h < TA / 128; ++h) {
      const int64_t x0 = a0 + h * 128;
      if (O.g) {
        // rows of G: queries; four consecutive rows of x are 8 bytes of it
        if (IB == 2 || wa == h) {
#pragma unroll
          for (int jb = 0; jb < JB; ++jb)
#pragma unroll
            for (int ib = 0; ib < IB; ++ib)
#pragma unroll
              for (int r = 0; r < 16; r += 4) {
                f16x4 v;
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = (_Float16)acc[ib][jb][r + u];
                *reinterpret_cast<f16x4*>(lds + ((wb * JB + jb) * 32 + (lane & 31)) * LDG +
                                          2 * ((IB == 2 ? wa * 64 : 0) + ib * 32 + 2 * r + 4 * half)) = v;
              }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < TB * 16; i += 256) {
          const int row = i >> 4, k = (i & 15) * 8;                 // 8 elements
          if (b0 + row < S.nq)
            *reinterpret_cast<u32x4*>(static_cast<char*>(O.g) + (b0 + row) * O.g_row_bytes + (x0 + k) / PER * 64 + plane * 32 +
                                      (k % PER) * 2) = *reinterpret_cast<const u32x4*>(lds + row * LDG + 2 * k);
        }
        __syncthreads();
      }
      if (O.gt) {
        if (IB == 2 || wa == h) {
#pragma unroll
          for (int jb = 0; jb < JB; ++jb)
#pragma unroll
            for (int ib = 0; ib < IB; ++ib)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                *reinterpret_cast<_Float16*>(lds + ((IB == 2 ? wa * 64 : 0) + ib * 32 + (r & 3) + 8 * (r >> 2) + 4 * half) * LDT +
                                             2 * ((wb * JB + jb) * 32 + (lane & 31))) = (_Float16)acc[ib][jb][r];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 128 * (TB / 8); i += 256) {
          const int row = i / (TB / 8), k = i % (TB / 8) * 8;
          if (x0 + row < S.nx)
            *reinterpret_cast<u32x4*>(static_cast<char*>(O.gt) + (x0 + row) * O.gt_row_bytes + (b0 + k) / PER * 64 + plane * 32 +
                                      (k % PER) * 2) = *reinterpret_cast<const u32x4*>(lds + row * LDT + 2 * k);
        }
        __syncthreads();
      }
    }
    if (PLANES == 2 && plane == 0) {
#pragma unroll
      for (int jb = 0; jb < JB; ++jb)
#pragma unroll
        for (int ib = 0; ib < IB; ++ib)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[ib][jb][r] -= (float)(_Float16)acc[ib][jb][r];
    }
  }
}

// Four elements at index i of an array of the vectors' type, the first n of them; whole: together (i a multiple of 4)
template <typename T>
__device__ __forceinline__ void store_4_as(T* p, int n, bool whole, const float (&v)[4]) {
  if (whole) {
    T e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) e[u] = (T)v[u];
    __builtin_memcpy(p, e, sizeof(e));
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (u < n) p[u] = (T)v[u];
  }
}
__device__ __forceinline__ void store_4(void* p, int64_t i, int n, bool whole, int dtype, const float (&v)[4]) {
  if (dtype == 0) store_4_as(static_cast<float*>(p) + i, n, whole, v);
  else if (dtype == 1) store_4_as(static_cast<_Float16*>(p) + i, n, whole, v);
  else store_4_as(static_cast<__bf16*>(p) + i, n, whole, v);
}

// ---- long products -------------------------------------------------------------------------
// out[b][a] = sum_k A[a][k] B[b][k] over long K: tiles of 256 x 256, eight wavefronts of 128 x 64 each.  Against 128 x 128
// tiles a K block reads three quarters of the LDS per product, and its 2048 cycles of products a SIMD cover the way of the
// next block from the last-level cache.  Fragments of the next 16 K elements are read while the present ones multiply.
// 768 x 4096 over K = 16,384 in 5 splits 145 us, 768 x 16,384 over K = 4096 142 us: 710 and 725 TFLOP/s.
constexpr int kBigTile = 256;
constexpr int kBigStage = 2 * kBigTile * 128;
// With one split and nothing to add to, results go out at once: out[b][a] = alpha sa[a] sum in the vectors' type, zeros
// where row b does not exist (bias -inf): zeros of G may have met a query that is not finite.
template <int PLANES, bool DIRECT>
__global__ __launch_bounds__(512, 1) void sm_product_kernel(SmMatrix A, SmMatrix B, int64_t kblocks, int splits, int add,
                                                            float* __restrict__ part, int64_t ld, int64_t ta, int64_t tb,
                                                            const float* __restrict__ sa, float alpha, int dtype, int d,
                                                            const float* __restrict__ bias) {
  extern __shared__ __align__(16) char lds[];
  int64_t ia, ib_;
  const int64_t tiles = ta * tb;
  const int split = (int)(blockIdx.x / tiles);
  tile_of(blockIdx.x - split * tiles, ta, tb, &ia, &ib_);
  const int64_t a0 = ia * kBigTile, b0 = ib_ * kBigTile;
  const int64_t k0 = kblocks * split / splits, k1 = kblocks * (split + 1) / splits;
  const int lane = lane_id(), wave = wave_id(), wa = wave & 1, wb = wave >> 1, half = lane >> 5;
  f32x16 acc[4][2] = {};
  float row_bias[2] = {0.f, 0.f};                     // (asked for before the sums: behind them every store would wait for it)
  if (DIRECT && bias) {
#pragma unroll
    for (int jb = 0; jb < 2; ++jb) {
      const int64_t b = b0 + wb * 64 + jb * 32 + (lane & 31);
      row_bias[jb] = bias[b < B.rows ? b : B.rows - 1];
    }
  }
  const char* pa = static_cast<const char*>(A.p) + a0 * A.row_bytes;
  const char* pb = static_cast<const char*>(B.p) + b0 * B.row_bytes;
  const int ra_max = (int)(A.rows - 1 - a0 < kBigTile ? A.rows - 1 - a0 : kBigTile - 1);
  const int rb_max = (int)(B.rows - 1 - b0 < kBigTile ? B.rows - 1 - b0 : kBigTile - 1);
  const char* ga[4];
  const char* gb[4];
  const int piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = (wave * 4 + i) * 8 + (lane >> 3);
    ga[i] = pa + (int64_t)(r < ra_max ? r : ra_max) * A.row_bytes + k0 * 128 + piece * 16;
    gb[i] = pb + (int64_t)(r < rb_max ? r : rb_max) * B.row_bytes + k0 * 128 + piece * 16;
  }
  auto request = [&](int stage) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)ga[i],
                                       (__attribute__((address_space(3))) void*)(lds + stage * kBigStage + (wave * 4 + i) * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)gb[i],
                                       (__attribute__((address_space(3))) void*)(lds + stage * kBigStage + kBigStage / 2 + (wave * 4 + i) * 1024), 16, 0, 0);
      ga[i] += 128;
      gb[i] += 128;
    }
  };
  const int ra = (wa * 128 + (lane & 31)) * 128, rb = (wb * 64 + (lane & 31)) * 128, sw = lane & 7;
  const int n = (int)(k1 - k0);
  if (n > 0) request(0);
  for (int t = 0; t < n; ++t) {
    __syncthreads();                                  // the stage has landed, the other one is free
    if (t + 1 < n) request((t + 1) & 1);
    const char* s = lds + (t & 1) * kBigStage;
    u32x4 a[2][4], b[2][2];
    auto fragments = [&](int ks, u32x4 (&fa)[4], u32x4 (&fb)[2]) {
      const int off = ((2 * ks + half) ^ sw) * 16;
#pragma unroll
      for (int ib = 0; ib < 4; ++ib) fa[ib] = *reinterpret_cast<const u32x4*>(s + ra + ib * 32 * 128 + off);
#pragma unroll
      for (int jb = 0; jb < 2; ++jb) fb[jb] = *reinterpret_cast<const u32x4*>(s + kBigStage / 2 + rb + jb * 32 * 128 + off);
    };
    auto products = [&](const u32x4 (&fa)[4], const u32x4 (&fb)[2]) {
#pragma unroll
      for (int ib = 0; ib < 4; ++ib)
#pragma unroll
        for (int jb = 0; jb < 2; ++jb) acc[ib][jb] = TileMul<PLANES, false>::mul(fa[ib], fb[jb], acc[ib][jb]);
    };
    if constexpr (PLANES == 1) {
      fragments(0, a[0], b[0]);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        if (ks < 3) fragments(ks + 1, a[(ks + 1) & 1], b[(ks + 1) & 1]);
        products(a[ks & 1], b[ks & 1]);
      }
    } else {                                          // two units of heads and tails: hi hi + hi lo + lo hi
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        fragments(2 * ks, a[0], b[0]);
        fragments(2 * ks + 1, a[1], b[1]);
        products(a[0], b[0]);
        products(a[0], b[1]);
        products(a[1], b[0]);
      }
    }
  }
  settle_products();
#pragma unroll
  for (int jb = 0; jb < 2; ++jb) {
    const int64_t b = b0 + wb * 64 + jb * 32 + (lane & 31);
    if (b >= B.rows) continue;
    if constexpr (DIRECT) {
      const bool gone = row_bias[jb] == neg_inf();
#pragma unroll
      for (int ib = 0; ib < 4; ++ib)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int a = (int)a0 + wa * 128 + ib * 32 + 2 * r + 4 * half;
          if (a >= d) continue;
          float v[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            v[u] = a + u < d ? acc[ib][jb][r + u] * sa[a + u] * alpha : 0.f;
            v[u] = gone ? 0.f : v[u];
          }
          store_4(part, b * d + a, d - a, (d & 3) == 0, dtype, v);
        }
      continue;
    }
    float* out = part + (split * B.rows + b) * ld;
#pragma unroll
    for (int ib = 0; ib < 4; ++ib)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int64_t a = a0 + wa * 128 + ib * 32 + 2 * r + 4 * half;
        if (a >= ld) continue;                                      // (ld is a multiple of 4 and at least A.rows)
        float4 v = make_float4(acc[ib][jb][r], acc[ib][jb][r + 1], acc[ib][jb][r + 2], acc[ib][jb][r + 3]);
        float4* o = reinterpret_cast<float4*>(out + a);
        if (add) { const float4 w = *o; v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w; }
        *o = v;
      }
  }
}

// The same on tiles of 128 x 64, for products that give 256 x 256 tiles too few workgroups.  K in units.
template <int PLANES>
__global__ __launch_bounds__(256, 2) void sm_product_small_kernel(SmMatrix A, SmMatrix B, int64_t kunits, int splits, int add,
                                                                  float* __restrict__ part, int64_t ld, int64_t ta, int64_t tb) {
  extern __shared__ __align__(16) char lds[];
  int64_t ia, ib_;
  const int64_t tiles = ta * tb;
  const int split = (int)(blockIdx.x / tiles);
  tile_of(blockIdx.x - split * tiles, ta, tb, &ia, &ib_);
  constexpr int IB = 2, JB = 1;
  const int64_t a0 = ia * 64 * IB, b0 = ib_ * 64 * JB;
  const int64_t k0 = kunits * split / splits, k1 = kunits * (split + 1) / splits;
  f32x16 acc[IB][JB] = {};
  if (k1 > k0) TileMul<PLANES, false, IB, JB>::run(A, a0, B, b0, k0, k1, lds, acc);
  const int lane = lane_id(), wave = wave_id(), wa = wave & 1, wb = wave >> 1, half = lane >> 5;
#pragma unroll
  for (int jb = 0; jb < JB; ++jb) {
    const int64_t b = b0 + (wb * JB + jb) * 32 + (lane & 31);
    if (b >= B.rows) continue;
    float* out = part + (split * B.rows + b) * ld;
#pragma unroll
    for (int ib = 0; ib < IB; ++ib)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int64_t a = a0 + (wa * IB + ib) * 32 + 2 * r + 4 * half;
        if (a >= ld) continue;
        float4 v = make_float4(acc[ib][jb][r], acc[ib][jb][r + 1], acc[ib][jb][r + 2], acc[ib][jb][r + 3]);
        float4* o = reinterpret_cast<float4*>(out + a);
        if (add) { const float4 w = *o; v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w; }
        *o = v;
      }
  }
}

template <int DT>
__global__ __launch_bounds__(256) void sm_product_out_kernel(const float* __restrict__ part, int splits, int64_t rows,
                                                             int64_t ld, int d, const float* __restrict__ sa,
                                                             const float* __restrict__ sb, float alpha,
                                                             const float* __restrict__ bias,
                                                             typename Elem<DT>::T* __restrict__ out) {
  const int64_t i = group_id() * 256 + threadIdx.x;
  if (i >= rows * d) return;
  const int64_t b = i / d;
  const int a = (int)(i - b * d);
  float v = 0.f;
  for (int s = 0; s < splits; ++s) v += part[(s * rows + b) * ld + a];
  // (powers of two first: the product with alpha is the only rounding before the last)
  v = v * sa[a] * (sb ? sb[b] : 1.f);
  if (bias && bias[b] == neg_inf()) v = 0.f;              // (a row that does not exist: see sm_product_kernel)
  out[i] = (typename Elem<DT>::T)(v * alpha);
}

__global__ __launch_bounds__(64) void sm_sum_parts_kernel(const float* __restrict__ part, int64_t parts, int64_t ld,
                                                           int64_t n, float* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x;
  if (i >= n) return;
  float v = 0.f;
#pragma unroll 8
  for (int64_t p = 0; p < parts; ++p) v += part[p * ld + i];
  out[i] = v;
}

__global__ __launch_bounds__(256) void sm_zero_kernel(u32* __restrict__ p, int64_t words) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) p[i] = 0;
}
__global__ __launch_bounds__(64) void sm_zero_bytes_kernel(unsigned char* __restrict__ p, int n) {
  if ((int)threadIdx.x < n) p[threadIdx.x] = 0;
}

inline int64_t tiles(int64_t n, int per) { return (n + per - 1) / per; }
inline unsigned grid_of(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

}  // namespace

void launch_sm_zero(void* p, int64_t bytes, hipStream_t st) {
  const int64_t words = bytes / 4;
  if (words > 0) {
    const unsigned g = grid_of(words, 256);
    sm_zero_kernel<<<g < 4096u ? g : 4096u, 256, 0, st>>>(static_cast<u32*>(p), words);
  }
  if (bytes & 3) sm_zero_bytes_kernel<<<1, 64, 0, st>>>(static_cast<unsigned char*>(p) + words * 4, (int)(bytes & 3));
}

void launch_sm_prep_rows(const SmForm& f, const SmSide& a, const SmSide& b, int d, hipStream_t st) {
  const int64_t dp = f.blocks(d) * f.per_block();
  const unsigned ga = grid_of(a.n, 16), n = ga + grid_of(b.n, 16);
  if (n == 0) return;
  const dim3 g = grid_2d(n);
  if (f.dtype == 0) sm_prep_rows_kernel<0, 2><<<g, 256, 0, st>>>(a, b, ga, d, dp);
  else if (f.dtype == 1) sm_prep_rows_kernel<1, 1><<<g, 256, 0, st>>>(a, b, ga, d, dp);
  else sm_prep_rows_kernel<2, 1><<<g, 256, 0, st>>>(a, b, ga, d, dp);
}

namespace {
template <int DT, int PLANES>
void prep_cols(SmSide a, SmSide b, const SmForm& f, int d, hipStream_t st) {
  typedef typename Elem<DT>::T T;
  a.np = f.blocks(a.n) * f.per_block();
  b.np = f.blocks(b.n) * f.per_block();
  const int64_t most = a.n > b.n ? a.n : b.n;
  const int64_t per = most < 64 * 1024 ? 64 : (most + 1023) / 1024;
  const unsigned ya = grid_of(a.n, (int)per), y = ya + grid_of(b.n, (int)per);
  sm_colmax_kernel<DT><<<dim3(grid_of(d, 64 * 16 / (int)sizeof(T)), y), 256, 0, st>>>(a, b, ya, d, per);
  const unsigned xa = grid_of(a.np, 64), x = xa + grid_of(b.np, 64);
  const dim3 g = grid_2d(x);
  sm_prep_cols_kernel<DT, PLANES><<<dim3(g.x, grid_of(d, 64), g.y), 256, 0, st>>>(a, b, xa, d);
}
}  // namespace

void launch_sm_prep_cols(const SmForm& f, const SmSide& a, const SmSide& b, int d, hipStream_t st) {
  if (a.n == 0 && b.n == 0) return;
  if (f.dtype == 0) prep_cols<0, 2>(a, b, f, d, st);
  else if (f.dtype == 1) prep_cols<1, 1>(a, b, f, d, st);
  else prep_cols<2, 1>(a, b, f, d, st);
}

void launch_sm_scores(const SmForm& f, bool direct, const SmScores& s, const SmRecords& r, bool second, hipStream_t st) {
  const int64_t ta = tiles(s.nx, kTileA), tb = tiles(s.nq, kTileB);
  const unsigned g = (unsigned)(ta * tb);
  auto run = [&](auto kern) { kern<<<g, 256, tile_lds<4, 2>(), st>>>(s, r, ta, tb); };
  if (f.planes == 2) { if (second) run(sm_scores_kernel<2, false, true>); else run(sm_scores_kernel<2, false, false>); }
  else if (direct && f.dtype == 2) { if (second) run(sm_scores_kernel<1, true, true>); else run(sm_scores_kernel<1, true, false>); }
  else { if (second) run(sm_scores_kernel<1, false, true>); else run(sm_scores_kernel<1, false, false>); }
}

namespace {
template <int DT, int NT>
void scores_few(const void* x, int64_t nb, const void* q, int64_t nq, int d, float scale, const float* bias,
                const SmRecords& r, bool second, hipStream_t st) {
  typedef typename Elem<DT>::T T;
  const dim3 g = grid_2d(r.parts);
  const int chunk = few_chunk<DT, NT>(), steps = ((d < chunk ? d : chunk) + FewMul<DT>::KS - 1) / FewMul<DT>::KS;
  const int recs = 4 * NT * 16 * 20, frags = steps * NT * 1024, lds = frags > recs ? frags : recs;
  if (second)
    sm_scores_few_kernel<DT, NT, true><<<g, 256, lds, st>>>(static_cast<const T*>(x), nb, static_cast<const T*>(q), (int)nq, d, scale, bias, r);
  else
    sm_scores_few_kernel<DT, NT, false><<<g, 256, lds, st>>>(static_cast<const T*>(x), nb, static_cast<const T*>(q), (int)nq, d, scale, bias, r);
}
}  // namespace

void launch_sm_scores_few(int dtype, const void* x, int64_t nb, const void* q, int64_t nq, int d, float scale,
                          const float* bias, const SmRecords& r, bool second, hipStream_t st) {
  if (nb == 0) return;
#define FEW(DT)                                                                          \
  do {                                                                                   \
    if (nq <= 16) scores_few<DT, 1>(x, nb, q, nq, d, scale, bias, r, second, st);        \
    else if (nq <= 32) scores_few<DT, 2>(x, nb, q, nq, d, scale, bias, r, second, st);   \
    else scores_few<DT, 4>(x, nb, q, nq, d, scale, bias, r, second, st);                 \
  } while (0)
  if (dtype == 0) FEW(0);
  else if (dtype == 1) FEW(1);
  else FEW(2);
#undef FEW
}

void launch_sm_finish(const SmFinish& f, const SmRecords& r, hipStream_t st) {
  const dim3 g = grid_2d(f.nq);
  const bool take = f.k <= kTakeBest && r.parts <= 256 * kTakePer && !r.keep;
  auto run = [&](auto some, auto all) {
    if (take) some<<<g, 256, 0, st>>>(f, r);
    else all<<<g, 256, 0, st>>>(f, r);
  };
  if (f.dtype == 0) run(sm_finish_kernel<0, true>, sm_finish_kernel<0, false>);
  else if (f.dtype == 1) run(sm_finish_kernel<1, true>, sm_finish_kernel<1, false>);
  else run(sm_finish_kernel<2, true>, sm_finish_kernel<2, false>);
}

void launch_sm_coefs(const SmGrads& g, int64_t nq, int64_t nb, float4* coef, float* bound, u32* clear, int n_clear, hipStream_t st) {
  sm_coefs_kernel<<<grid_of(nq, 256), 256, 0, st>>>(g, nq, nb, coef, bound, clear, n_clear);
}

// Tiles of 128 x 64 pairs or of 256 x 128.  A pair's epilogue (its probability, the two G) costs as much as some 400 of
// its products, and four small workgroups on a CU hide it behind each other's products where two big ones do not; what
// the big ones save is operand traffic, which counts with one plane and long rows.  Small and big in us: fp32 1024 x 1024
// x 96 59 and 83, bf16 65,536 x 4096: d = 128 946 and 1031, 384 1488 and 1545, 768 2051 and 2010; fp32 16,384 x 4096 x 768
// 1398 and 1484; bf16 8192 x 2048 x 768 221 and 217, 4096 x 1024 x 768 (128 big tiles for 256 CUs) 109 and 111.
bool sm_gradients_small(const SmForm& f, int64_t nx, int64_t nq, int64_t kblocks) {
  return f.planes == 2 || kblocks < 10 || tiles(nx, kTileA) * tiles(nq, kTileB) < 256;
}

void launch_sm_gradients(const SmForm& f, bool direct, const SmScores& s, const SmGOut& o, hipStream_t st) {
  auto run = [&](auto kern, int ib, int jb, int lds) {
    const int64_t ta = tiles(s.nx, 64 * ib), tb = tiles(s.nq, 64 * jb);
    kern<<<(unsigned)(ta * tb), 256, lds, st>>>(s, o, ta, tb);
  };
  if (o.small) {
    constexpr int lds = 64 * (2 * 128 + 16) > 128 * (2 * 64 + 16) ? 64 * (2 * 128 + 16) : 128 * (2 * 64 + 16);
    const int n = tile_lds<2, 1>() > lds ? tile_lds<2, 1>() : lds;
    if (f.planes == 2) run(sm_gradients_kernel<2, false, 2, 1>, 2, 1, n);
    else if (direct && f.dtype == 2) run(sm_gradients_kernel<1, true, 2, 1>, 2, 1, n);
    else run(sm_gradients_kernel<1, false, 2, 1>, 2, 1, n);
  } else {
    const int n = tile_lds<4, 2>();                       // (one plane: sm_gradients_small)
    if (direct && f.dtype == 2) run(sm_gradients_kernel<1, true, 4, 2>, 4, 2, n);
    else run(sm_gradients_kernel<1, false, 4, 2>, 4, 2, n);
  }
}

// Splits of K that give a product some 256 workgroups, eight 128-byte blocks each at least.  big: tiles of 256 x 256, where
// they fill the CUs by themselves or K is long enough to split.  Whole gradients on big and on small tiles in us: bf16
// 65,536 x 4096 x 768 (768 big tiles for dx, 48 with 1024 blocks of K for dq) 2010 and 2591, 65,536 x 4096 x 128 (256 tiles)
// 1031 and 1077, fp16 30,011 x 777 x 400 (236) 241 and 275; 30,011 x 777 x 100 (118) 169 and 163, bf16 8192 x 2048 x 768
// (96, 32 blocks of K) 217 and 201, 4096 x 1024 x 768 (48) 111 and 103.
SmProductPlan plan_sm_product(int64_t rows_a, int64_t rows_b, int64_t kblocks) {
  SmProductPlan p;
  const int64_t big = (rows_a + kBigTile - 1) / kBigTile * ((rows_b + kBigTile - 1) / kBigTile);
  p.big = big >= 160 || (big >= 48 && kblocks >= 256);
  const int64_t n = p.big ? big : tiles(rows_a, 128) * tiles(rows_b, 64), most = kblocks / (p.big ? 8 : 4);
  int64_t want = p.big ? (256 + n / 2) / n : (512 + n - 1) / n;
  if (want > most) want = most;
  if (want > 16) want = 16;
  p.splits = want < 1 ? 1 : (int)want;
  p.groups = n * p.splits;
  return p;
}

void launch_sm_product(const SmForm& f, const SmProductPlan& pp, const SmMatrix& A, const SmMatrix& B, int64_t kblocks, bool add,
                       float* part, int64_t ld, hipStream_t st) {
  if (pp.big) {
    const int64_t ta = (A.rows + kBigTile - 1) / kBigTile, tb = (B.rows + kBigTile - 1) / kBigTile;
    const unsigned g = (unsigned)(ta * tb * pp.splits);
    auto run = [&](auto kern) {
      (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kBigStage);
      kern<<<g, 512, 2 * kBigStage, st>>>(A, B, kblocks, pp.splits, add ? 1 : 0, part, ld, ta, tb, nullptr, 0.f, 0, 0, nullptr);
    };
    if (f.planes == 2) run(sm_product_kernel<2, false>);
    else run(sm_product_kernel<1, false>);
  } else {
    const int64_t ta = tiles(A.rows, 128), tb = tiles(B.rows, 64);
    const unsigned g = (unsigned)(ta * tb * pp.splits);
    if (f.planes == 2) sm_product_small_kernel<2><<<g, 256, tile_lds<2, 1>(), st>>>(A, B, 2 * kblocks, pp.splits, add ? 1 : 0, part, ld, ta, tb);
    else sm_product_small_kernel<1><<<g, 256, tile_lds<2, 1>(), st>>>(A, B, 2 * kblocks, pp.splits, add ? 1 : 0, part, ld, ta, tb);
  }
}

void launch_sm_product_direct(const SmForm& f, const SmMatrix& A, const SmMatrix& B, int64_t kblocks, const float* sa,
                              float alpha, const float* bias, int dtype, void* out, hipStream_t st) {
  const int64_t ta = (A.rows + kBigTile - 1) / kBigTile, tb = (B.rows + kBigTile - 1) / kBigTile;
  const unsigned g = (unsigned)(ta * tb);
  auto run = [&](auto kern) {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kBigStage);
    kern<<<g, 512, 2 * kBigStage, st>>>(A, B, kblocks, 1, 0, static_cast<float*>(out), 0, ta, tb, sa, alpha, dtype, (int)A.rows, bias);
  };
  if (f.planes == 2) run(sm_product_kernel<2, true>);
  else run(sm_product_kernel<1, true>);
}

void launch_sm_product_out(const float* part, int splits, int64_t rows, int64_t ld, int d, const float* sa, const float* sb,
                           float alpha, const float* bias, int dtype, void* out, hipStream_t st) {
  const dim3 g = grid_2d((rows * d + 255) / 256);
  if (dtype == 0) sm_product_out_kernel<0><<<g, 256, 0, st>>>(part, splits, rows, ld, d, sa, sb, alpha, bias, static_cast<float*>(out));
  else if (dtype == 1) sm_product_out_kernel<1><<<g, 256, 0, st>>>(part, splits, rows, ld, d, sa, sb, alpha, bias, static_cast<_Float16*>(out));
  else sm_product_out_kernel<2><<<g, 256, 0, st>>>(part, splits, rows, ld, d, sa, sb, alpha, bias, static_cast<__bf16*>(out));
}

void launch_sm_sum_parts(const float* part, int64_t n_parts, int64_t ld, int64_t n, float* out, hipStream_t st) {
  sm_sum_parts_kernel<<<grid_of(n, 64), 64, 0, st>>>(part, n_parts, ld, n, out);
}
