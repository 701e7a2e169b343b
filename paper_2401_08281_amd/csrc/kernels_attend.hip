// Attention over the vectors of a 4-bit IVF-PQ index, and its gradient for the queries.
//
// Both products of attention are taken in the code domain.  With keys and values x'_j = c_l + concat_m T_m[code_jm]:
//   s_ij  = scale <q, c_l> + sum_m LUT_m[code_jm],  LUT_m[c] = scale <q_m, T_m[c]>            (a look-up per sub-quantizer)
//   out_i = sum_l P_l c_l + concat_m sum_c H_m[c] T_m[c],  H_m[c] = sum of p_j with code_jm = c  (an addition per one)
// so a stored vector costs 2 M operations on LDS a query instead of 2 d products, whatever its dimension.
//
// A workgroup takes QB queries and a part of the rows, in rounds of up to 2048 rows: scores (one row a lane, all
// queries), their maximum, weights, then the weighted sums (one sub-quantizer a lane).  Codewords of up to four components
// are looked up whole and added to the lane's registers; longer ones go through the histograms H: a lane adds to its own
// column of its wavefront's H only, so additions keep their order and banks never collide.  (Additions by LDS atomics ran
// at 24 cycles a wavefront, three times the whole scan.)  Partial results of the parts are joined by a second kernel.
// Bound by LDS: one look-up of QB values, and one of a codeword or a histogram cell, for every code.  1000 queries x 7812
// codes of 64 sub-quantizers (histograms) 460 us, 2.2 look-ups a ns; gradient of 333 queries x 3200 codes of 32 (codewords)
// 81 us, 1.3; one query x 4097 codes 21 us, its set-up and two rounds.
#include <algorithm>

#include "../../include/vs_softmax.h"
#include "common.hpp"
#include "softmax.hpp"

namespace {

typedef u32 u32x2 __attribute__((ext_vector_type(2)));
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kRound = 2048;        // rows of a round
constexpr int kSegments = 64;       // lists it may span
constexpr int kTiles = kRound / 64 + kSegments;   // runs of up to 64 rows of one list
constexpr int kWaves = 4;
constexpr int kCodeRun = 72;        // bytes of a staged run of 64 rows' codes (18 words: runs start in different banks)
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) v = fmaxf(v, __shfl_xor(v, w));
  return v;
}
__device__ __forceinline__ float load_as_f32(const void* p, int64_t i, int dtype) {
  if (dtype == VS_FP32) return static_cast<const float*>(p)[i];
  if (dtype == VS_FP16) return (float)static_cast<const _Float16*>(p)[i];
  return (float)static_cast<const __bf16*>(p)[i];
}
__device__ __forceinline__ void store_as(void* p, int64_t i, int dtype, float v) {
  if (dtype == VS_FP32) static_cast<float*>(p)[i] = v;
  else if (dtype == VS_FP16) static_cast<_Float16*>(p)[i] = (_Float16)v;
  else static_cast<__bf16*>(p)[i] = (__bf16)v;
}

struct ScanArgs {
  IvfpqDims g;
  const float* centroids;
  const float* codebooks;
  const uint8_t* codes;
  const int64_t* ids;
  const int64_t* list_off;
  int64_t ntotal;
  const void* q; int64_t nq; int dk, v0, dtype; float scale;
  const int64_t* limits;
  const int32_t* probes; int nprobe;      // null: all lists
  int nsplit; int64_t per;                // parts of a query's rows; rows (probes, if any) of a part
  const float* lse; const void* g_out;    // backward
  float* part;                            // [nq][nsplit][ld]: {max, sum, out}, or with w = p (dp - shift) {sum w, sum p, shift, sum w k, sum p k}
  int64_t ld;
};

// Rows [first, first + len) of a round; first is a multiple of eight, and weights up to the next one are zero.
struct Segment { int64_t pos; int32_t list, first, len, pad; };
struct Tile { int64_t pos; int32_t first, len_seg; };              // a run: length, segment << 8

// Groups of lanes that a wavefront's 64 rows are shared out to: 1, 2, 4 or 8 (eight rows each at least)
__device__ __forceinline__ int row_groups(int mh) { return mh > 32 ? 1 : (mh > 16 ? 2 : (mh > 8 ? 4 : 8)); }

// What a workgroup of QB queries keeps in LDS, in floats.
struct ScanLds {
  int lut, lut2, q, g, score, score2, hist, words, cacc, codes, bias, bias2, red, seg, tiles, total;
  int mh, mc;                        // histogrammed sub-quantizers; 64-lane chunks of them
};
// Components of a looked-up codeword, padded (0: histograms): where a lane holds one sub-quantizer and 16 bytes hold one
__host__ __device__ inline int scan_words(const IvfpqDims& g, int dk, int v0, bool grad) {
  const int mh = (grad ? dk : g.d - v0) / g.dsub;
  return mh > 64 || g.dsub > 4 ? 0 : (g.dsub > 2 ? 4 : g.dsub);
}
__host__ __device__ inline ScanLds scan_lds(const IvfpqDims& g, int dk, int v0, int qb, bool grad) {
  ScanLds o{};
  const int mk = dk / g.dsub, mv = (g.d - v0) / g.dsub, out = grad ? dk : g.d - v0, sets = grad ? 2 : 1;
  o.mh = grad ? mk : mv;
  o.mc = (o.mh + 63) / 64;
  int at = 0;
  auto take = [&](int n) { const int o2 = at; at += (n + 3) / 4 * 4; return o2; };
  o.lut = take(mk * 16 * qb);
  o.lut2 = take(grad ? mv * 16 * qb : 0);
  o.q = take(dk * qb);
  o.g = take(grad ? (g.d - v0) * qb : 0);
  o.score = take(kRound * qb);
  o.score2 = take(grad ? kRound * qb : 0);
  const int ds = scan_words(g, dk, v0, grad);
  o.hist = take(ds ? 0 : kWaves * sets * qb * o.mc * 1024);
  o.words = take(16 * o.mh * ds);
  o.cacc = take(sets * qb * out);
  o.codes = take((kWaves * g.code_size * kCodeRun + 3) / 4);
  o.bias = take(kSegments * qb);
  o.bias2 = take(grad ? kSegments * qb : 0);
  o.red = take(kWaves * 2 * qb + 8);
  o.seg = take((int)(sizeof(Segment) / 4) * kSegments + 8);
  o.tiles = take((int)(sizeof(Tile) / 4) * kTiles);
  o.total = at;
  return o;
}

// Words of a code row of cs bytes, the last one filled up with zeros.
__device__ __forceinline__ u32 code_word(const uint8_t* row, int w, int cs) {
  u32 v = 0;
  if (4 * w + 4 <= cs) {
    __builtin_memcpy(&v, row + 4 * w, 4);
  } else {
    for (int b = 4 * w; b < cs; ++b) v |= (u32)row[b] << (8 * (b & 3));
  }
  return v;
}

template <int QB>
__device__ __forceinline__ void look_up(const float* lut, u32 word, int u, float (&acc)[QB]) {
  const float* e = lut + (u * 16 + ((word >> (4 * u)) & 15u)) * QB;
  if constexpr (QB == 2) {
    const float2 v = *reinterpret_cast<const float2*>(e);
    acc[0] += v.x;
    acc[1] += v.y;
  } else {
    acc[0] += e[0];
  }
}
// The words of a row, requested together (rows of up to 64 bytes; longer ones are read as they are used)
constexpr int kRowWords = 16;
__device__ __forceinline__ void load_row(const uint8_t* row, int cs, u32 (&w)[kRowWords]) {
  if ((cs & 15) == 0) {
#pragma unroll
    for (int i = 0; i < kRowWords; i += 4) {
      u32x4 v = {0, 0, 0, 0};
      if (i * 4 < cs) __builtin_memcpy(&v, row + i * 4, 16);
      w[i] = v[0]; w[i + 1] = v[1]; w[i + 2] = v[2]; w[i + 3] = v[3];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kRowWords; ++i) w[i] = i * 4 < cs ? code_word(row, i, cs) : 0u;
  }
}

// Sum of the look-ups of sub-quantizers [m0, m1) of one row, in two chains: half the roundings in a row, and no addition
// waits for the one before.  The bias, usually the largest term, comes last.
template <int QB>
__device__ __forceinline__ void score_word(u32 word, int w, int m0, int m1, const float* lut, float (&acc)[2][QB]) {
  const float* t = lut + (w * 8 - m0) * 16 * QB;
  if (w * 8 >= m0 && w * 8 + 8 <= m1) {
#pragma unroll
    for (int u = 0; u < 8; ++u) look_up<QB>(t, word, u, acc[u & 1]);
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (w * 8 + u >= m0 && w * 8 + u < m1) look_up<QB>(t, word, u, acc[u & 1]);
  }
}
template <int QB>
__device__ __forceinline__ void score_row(const uint8_t* row, const u32 (&words)[kRowWords], int cs, int m0, int m1,
                                          const float* lut, const float* bias, float (&out)[QB]) {
  float acc[2][QB] = {};
  if (cs <= 4 * kRowWords) {
#pragma unroll
    for (int w = 0; w < kRowWords; ++w)
      if (w * 8 < m1 && w * 8 + 8 > m0) score_word<QB>(words[w], w, m0, m1, lut, acc);
  } else {
    for (int w = m0 / 8; w * 8 < m1; ++w) score_word<QB>(code_word(row, w, cs), w, m0, m1, lut, acc);
  }
#pragma unroll
  for (int b = 0; b < QB; ++b) out[b] = (acc[0][b] + acc[1][b]) + bias[b];
}

// N weights of consecutive rows (a multiple of 16 bytes from a multiple of 16 bytes on)
template <int N>
__device__ __forceinline__ void load_weights(const float* p, float (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = *reinterpret_cast<const float4*>(p + i);
    w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
  }
}

// Two rows' weights into one column of a histogram: both cells are read before either is written; where the codes are
// equal both writes carry the sum.
__device__ __forceinline__ void add_pair(float* h, u32 c0, u32 c1, float p0, float p1) {
  const float v0 = h[c0 * 64], v1 = h[c1 * 64];
  const float s0 = v0 + p0, s1 = (c0 == c1 ? s0 : v1) + p1;
  h[c0 * 64] = s0;
  h[c1 * 64] = s1;                          // (after the first: with equal codes this one stays)
}

template <int QB, bool GRAD, int DS>
__global__ __launch_bounds__(256) void attend_scan_kernel(ScanArgs A) {
  extern __shared__ __align__(16) float lds[];
  const ScanLds L = scan_lds(A.g, A.dk, A.v0, QB, GRAD);
  constexpr int SETS = GRAD ? 2 : 1;
  const int lane = lane_id(), wave = wave_id();
  const int d = A.g.d, dsub = A.g.dsub, M = A.g.M, cs = A.g.code_size, dv = d - A.v0;
  const int mk = A.dk / dsub, mv = dv / dsub, mv0 = M - mv;
  const int h0 = GRAD ? 0 : mv0, hd0 = GRAD ? 0 : A.v0, nout = GRAD ? A.dk : dv;   // the histogrammed sub-quantizers
  const u32 wg = (u32)group_id();                              // (below 2^31)
  const int split = wg % A.nsplit;
  const int64_t q0 = (int64_t)(wg / A.nsplit) * QB;
  if (q0 >= A.nq) return;
  Segment* segs = reinterpret_cast<Segment*>(lds + L.seg);
  int* ctl = reinterpret_cast<int*>(lds + L.seg + (int)(sizeof(Segment) / 4) * kSegments);   // {segments, rows, next candidate, -, offset (two words), runs}
  int64_t* offset = reinterpret_cast<int64_t*>(ctl + 4);         // rows of the next candidate that are done
  Tile* tiles = reinterpret_cast<Tile*>(lds + L.tiles);
  float* hist = lds + L.hist + wave * SETS * QB * L.mc * 1024;

  for (int i = threadIdx.x; i < QB * A.dk; i += 256) {
    const int64_t qi = q0 + i / A.dk;
    lds[L.q + i] = qi < A.nq ? load_as_f32(A.q, qi * A.dk + i % A.dk, A.dtype) * A.scale : 0.f;
  }
  if (GRAD)
    for (int i = threadIdx.x; i < QB * dv; i += 256) {
      const int64_t qi = q0 + i / dv;
      lds[L.g + i] = qi < A.nq ? load_as_f32(A.g_out, qi * dv + i % dv, A.dtype) : 0.f;
    }
  if (DS == 0)
    for (int i = threadIdx.x; i < kWaves * SETS * QB * L.mc * 1024; i += 256) lds[L.hist + i] = 0.f;
  // codewords [code][sub-quantizer][DS]: sixteen lanes of consecutive sub-quantizers never share a bank, whatever the codes
  for (int i = threadIdx.x; i < 16 * L.mh * DS; i += 256) {
    const int u = i % (DS > 0 ? DS : 1), m = i / (DS > 0 ? DS : 1) % L.mh, c = i / (DS > 0 ? DS : 1) / L.mh;
    lds[L.words + i] = u < dsub ? A.codebooks[((int64_t)(h0 + m) * 16 + c) * dsub + u] : 0.f;
  }
  for (int i = threadIdx.x; i < SETS * QB * nout; i += 256) lds[L.cacc + i] = 0.f;
  // the part's rows: candidates are its probes, or the lists that its rows lie in
  int64_t r0 = 0, r1 = 0;
  int c0, c_end;
  if (A.probes) {
    c0 = (int)(split * A.per);
    c_end = (int)(c0 + A.per < A.nprobe ? c0 + A.per : A.nprobe);
  } else {
    r0 = split * A.per;
    r1 = r0 + A.per < A.ntotal ? r0 + A.per : A.ntotal;
    c0 = r0 < r1 ? list_of_position(A.list_off, A.g.nlist, r0) : 0;
    c_end = r0 < r1 ? list_of_position(A.list_off, A.g.nlist, r1 - 1) + 1 : 0;
  }
  if (threadIdx.x == 0) { ctl[2] = c0; *offset = 0; }
  __syncthreads();
  for (int i = threadIdx.x; i < mk * 16; i += 256) {
    const float* t = A.codebooks + (int64_t)i * dsub;
    const int m = i >> 4;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      float s = 0.f;
      for (int u = 0; u < dsub; ++u) s = __builtin_fmaf(lds[L.q + b * A.dk + m * dsub + u], t[u], s);
      lds[L.lut + i * QB + b] = s;
    }
  }
  if (GRAD)
    for (int i = threadIdx.x; i < mv * 16; i += 256) {
      const float* t = A.codebooks + (int64_t)(mv0 * 16 + i) * dsub;
      const int m = i >> 4;
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        float s = 0.f;
        for (int u = 0; u < dsub; ++u) s = __builtin_fmaf(lds[L.g + b * dv + m * dsub + u], t[u], s);
        lds[L.lut2 + i * QB + b] = s;
      }
    }
  int64_t limit[QB];
  float lse[QB], mx[QB], sum[QB], sum2[QB], shift[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    const bool in = q0 + b < A.nq;
    limit[b] = !in ? INT64_MIN : (A.limits ? A.limits[q0 + b] : INT64_MAX);
    lse[b] = GRAD && in ? A.lse[q0 + b] : 0.f;
    if (GRAD && lse[b] == neg_inf()) limit[b] = INT64_MIN;      // saw nothing
    mx[b] = neg_inf(); sum[b] = 0.f; sum2[b] = 0.f; shift[b] = 0.f;
  }
  const int rstep = row_groups(L.mh), rs = lane / (L.mh < 64 ? L.mh : 64), hm = lane % (L.mh < 64 ? L.mh : 64);
  const bool hist_lane = rs < rstep && hm < L.mh;
  float word_sum[SETS][QB][DS > 0 ? DS : 1] = {};

  while (true) {
    __syncthreads();
    if (wave == 0) {                              // the segments of this round, a candidate list a lane
      const int next = ctl[2], c = next + lane;
      const int64_t off = *offset;
      int64_t b = 0, e = 0;
      int list = -1;
      if (c < c_end) {
        list = A.probes ? A.probes[q0 * A.nprobe + c] : c;
        if (list >= 0 && list < A.g.nlist) {
          b = A.list_off[list];
          e = A.list_off[list + 1];
          if (!A.probes) { b = b > r0 ? b : r0; e = e < r1 ? e : r1; }
          if (lane == 0) b += off;
        }
      }
      const int64_t have = e > b ? e - b : 0;
      const int len0 = (int)(have < kRound ? have : kRound);
      int end = (len0 + 7) & ~7;                  // inclusive prefix sum
      const int len8 = end;
#pragma unroll
      for (int w = 1; w < 64; w <<= 1) {
        const int o = __shfl_up(end, w);
        if (lane >= w) end += o;
      }
      const int first = end - len8;
      const int len = first >= kRound ? 0 : (len0 < kRound - first ? len0 : kRound - first);
      const u64 taken = __ballot(len > 0);
      int runs = (len + 63) / 64, run_end = runs;
#pragma unroll
      for (int w = 1; w < 64; w <<= 1) {
        const int o = __shfl_up(run_end, w);
        if (lane >= w) run_end += o;
      }
      if (len > 0) {
        const int at = __popcll(taken & ((1ull << lane) - 1));
        segs[at] = Segment{b, list, first, len, 0};
        for (int i = 0; i < runs; ++i)
          tiles[run_end - runs + i] = Tile{b + i * 64, first + i * 64, (len - i * 64 < 64 ? len - i * 64 : 64) | at << 8};
      }
      if (lane == 63) ctl[6] = run_end;
      // the next round starts at the first candidate that is not used up
      const u64 open = __ballot(c < c_end && have > len);
      const int stop = open ? __ffsll(open) - 1 : 64;
      if (lane == (stop < 64 ? stop : 63)) {
        ctl[0] = __popcll(taken);
        ctl[1] = end < kRound ? end : kRound;
        ctl[2] = next + stop;
        *offset = stop < 64 ? (stop == 0 ? off + len : len) : 0;
      }
    }
    __syncthreads();
    const int nseg = ctl[0], rows = ctl[1], next = ctl[2], ntile = ctl[6];
    if (nseg == 0) {
      if (next >= c_end) break;
      continue;
    }
    // biases of the segments' lists
    for (int s = wave; s < nseg; s += kWaves) {
      const float* c = A.centroids + (int64_t)segs[s].list * d;
      float v[QB] = {}, v2[QB] = {};
#pragma unroll 4
      for (int t = lane; t < A.dk; t += 64) {
        const float ct = c[t];
#pragma unroll
        for (int b = 0; b < QB; ++b) v[b] = __builtin_fmaf(lds[L.q + b * A.dk + t], ct, v[b]);
      }
      if (GRAD)
#pragma unroll 4
        for (int t = lane; t < dv; t += 64) {
          const float ct = c[A.v0 + t];
#pragma unroll
          for (int b = 0; b < QB; ++b) v2[b] = __builtin_fmaf(lds[L.g + b * dv + t], ct, v2[b]);
        }
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        v[b] = wave_sum(v[b]);
        if (GRAD) v2[b] = wave_sum(v2[b]);
        if (lane == 0) {
          lds[L.bias + s * QB + b] = v[b];
          if (GRAD) lds[L.bias2 + s * QB + b] = v2[b];
        }
      }
    }
    __syncthreads();
    // scores
    float top[QB], rp[QB], rw[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) { top[b] = neg_inf(); rp[b] = 0.f; rw[b] = 0.f; }
    // (the codes of a wavefront's next run are on their way while it looks up the present one)
    u32 words[kRowWords];
    int64_t id = 0;
    auto fetch = [&](int ti) {
      const Tile tl = tiles[ti];
      const int64_t pos = tl.pos + (lane < (tl.len_seg & 255) ? lane : 0);
      if (cs <= 4 * kRowWords) load_row(A.codes + pos * cs, cs, words);
      if (A.limits) id = A.ids[pos];
    };
    if (wave < ntile) fetch(wave);
    for (int ti = wave; ti < ntile; ti += kWaves) {
      const Tile tl = tiles[ti];
      const int s = tl.len_seg >> 8, i = tl.first + lane;
      u32 now[kRowWords];
#pragma unroll
      for (int w = 0; w < kRowWords; ++w) now[w] = words[w];
      const int64_t my_id = id;
      if (ti + kWaves < ntile) fetch(ti + kWaves);
      const int n = tl.len_seg & 255;
      if (lane >= n && lane < ((n + 7) & ~7)) {
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          lds[L.score + i * QB + b] = GRAD ? 0.f : neg_inf();
          if (GRAD) lds[L.score2 + i * QB + b] = 0.f;
        }
      }
      if (lane < n) {
        float acc[QB], acc2[QB];
        const uint8_t* row = A.codes + (tl.pos + lane) * cs;
        score_row<QB>(row, now, cs, 0, mk, lds + L.lut, lds + L.bias + s * QB, acc);
        if (GRAD) score_row<QB>(row, now, cs, mv0, M, lds + L.lut2, lds + L.bias2 + s * QB, acc2);
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          const bool sees = my_id < limit[b];
          if (GRAD) {
            const float p = sees ? exp_neg(acc[b] - lse[b]) : 0.f;
            const float w = sees ? p * acc2[b] : 0.f;
            lds[L.score + i * QB + b] = p;
            lds[L.score2 + i * QB + b] = acc2[b];
            rp[b] += p;
            rw[b] += w;
          } else {
            const float v = sees ? acc[b] : neg_inf();
            lds[L.score + i * QB + b] = v;
            top[b] = fmaxf(top[b], v);
          }
        }
      }
    }
    if (!GRAD) {                                  // weights under the running maximum
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        top[b] = wave_max(top[b]);
        if (lane == 0) lds[L.red + wave * QB + b] = top[b];
      }
      __syncthreads();
      bool grown = false;
      float f[QB];
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        float m = mx[b];
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, lds[L.red + w * QB + b]);
        f[b] = mx[b] == neg_inf() ? 1.f : exp_neg(mx[b] - m);      // (nothing yet: zeros to scale)
        grown |= f[b] != 1.f;
        mx[b] = m;
        sum[b] *= f[b];
      }
      if (grown) {
        if (DS == 0)
          for (int i = threadIdx.x; i < kWaves * QB * L.mc * 1024; i += 256) lds[L.hist + i] *= f[QB == 1 ? 0 : (i / (L.mc * 1024)) % QB];
#pragma unroll
        for (int b = 0; b < QB; ++b)
#pragma unroll
          for (int u = 0; u < (DS > 0 ? DS : 1); ++u) word_sum[0][b][u] *= f[b];
        for (int i = threadIdx.x; i < QB * nout; i += 256) lds[L.cacc + i] *= f[QB == 1 ? 0 : i / nout];
      }
      for (int i = threadIdx.x; i < rows * QB; i += 256) {
        const int b = QB == 1 ? 0 : i % QB;
        const float v = lds[L.score + i];
        const float p = v == neg_inf() ? 0.f : exp_neg(v - mx[b]);
        lds[L.score + i] = p;
        if (QB == 1) sum[0] += p; else if (b == 0) sum[0] += p; else sum[QB - 1] += p;
      }
    }
    if (GRAD) {
      // The sums of p dp k and (sum p dp) p k nearly cancel; taken relative to the mean of dp over the part's first round
      // with any weight they do not.
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        rp[b] = wave_sum(rp[b]);
        rw[b] = wave_sum(rw[b]);
        if (lane == 0) { lds[L.red + wave * 2 * QB + b] = rp[b]; lds[L.red + wave * 2 * QB + QB + b] = rw[b]; }
      }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        float p = 0.f, w = 0.f;
        for (int v = 0; v < kWaves; ++v) { p += lds[L.red + v * 2 * QB + b]; w += lds[L.red + v * 2 * QB + QB + b]; }
        if (!(mx[b] > neg_inf()) && p > 0.f) { shift[b] = w / p; mx[b] = 0.f; }      // (mx: whether the shift is set)
      }
      for (int i = threadIdx.x; i < rows * QB; i += 256) {
        const int b = QB == 1 ? 0 : i % QB;
        const float p = lds[L.score + i], w = p == 0.f ? 0.f : p * (lds[L.score2 + i] - (b == 0 ? shift[0] : shift[QB - 1]));
        lds[L.score2 + i] = w;
        if (b == 0) { sum[0] += p; sum2[0] += w; } else { sum[QB - 1] += p; sum2[QB - 1] += w; }
      }
    }
    __syncthreads();
    // centroids, weighted by their lists' sums
    for (int s = wave; s < nseg; s += kWaves) {
      const Segment sg = segs[s];
      float w[SETS][QB] = {};
      for (int i = lane; i < sg.len; i += 64)
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          w[SETS - 1][b] += lds[L.score + (sg.first + i) * QB + b];
          if (GRAD) w[0][b] += lds[L.score2 + (sg.first + i) * QB + b];
        }
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        w[SETS - 1][b] = wave_sum(w[SETS - 1][b]);
        if (GRAD) w[0][b] = wave_sum(w[0][b]);
        if (lane == 0) {
          lds[L.bias + s * QB + b] = w[SETS - 1][b];
          if (GRAD) lds[L.bias2 + s * QB + b] = w[0][b];
        }
      }
    }
    // histograms: a wavefront takes 64 rows, turns their codes round in LDS (byte m / 2 of 64 rows in a run) and adds them
    // eight rows at a time; its groups of lanes, if sub-quantizers leave room for several, take a part of the rows each
    if (wave < ntile) fetch(wave);
    for (int ti = wave; ti < ntile; ti += kWaves) {
      const Tile tl = tiles[ti];
      const int n = tl.len_seg & 255;
      {
        uint8_t* ct = reinterpret_cast<uint8_t*>(lds + L.codes) + wave * cs * kCodeRun;
        wave_lds_sync();
        if (cs <= 4 * kRowWords) {
#pragma unroll
          for (int w = 0; w < kRowWords; ++w)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (w * 4 + u < cs) ct[(w * 4 + u) * kCodeRun + lane] = (uint8_t)(words[w] >> (8 * u));
        } else {
          const uint8_t* row = A.codes + (tl.pos + (lane < n ? lane : 0)) * cs;
          for (int i = 0; i < cs; ++i) ct[i * kCodeRun + lane] = row[i];
        }
        if (ti + kWaves < ntile) fetch(ti + kWaves);
        wave_lds_sync();
        if (hist_lane) {
          const float* pr = lds + L.score + tl.first * QB;
          const float* pr2 = lds + L.score2 + tl.first * QB;
          const int per = 64 / rstep, j0 = rs * per, n8 = (n + 7) & ~7, j1 = n8 < j0 + per ? n8 : j0 + per;
          if constexpr (DS > 0) {
            typedef float words_t __attribute__((ext_vector_type(DS)));
            const uint8_t* cb = ct + (h0 + hm) / 2 * kCodeRun;
            const int sh = ((h0 + hm) & 1) * 4;
            const float* tab = lds + L.words + hm * DS;
            const u32 stride = L.mh * DS;
            for (int j = j0; j < j1; j += 8) {
              u32x2 c8 = *reinterpret_cast<const u32x2*>(cb + j);
              c8 >>= sh;
              words_t t[8];
#pragma unroll
              for (int i = 0; i < 8; ++i)
                t[i] = *reinterpret_cast<const words_t*>(tab + __umul24((c8[i >> 2] >> (8 * (i & 3))) & 15u, stride));
              float p[8 * QB], p2[8 * QB];
              load_weights<8 * QB>(pr + j * QB, p);
              if (GRAD) load_weights<8 * QB>(pr2 + j * QB, p2);
#pragma unroll
              for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int b = 0; b < QB; ++b)
#pragma unroll
                  for (int u = 0; u < DS; ++u) {
                    const float w = t[i][u];
                    if (GRAD) word_sum[0][b][u] = __builtin_fmaf(p2[i * QB + b], w, word_sum[0][b][u]);
                    word_sum[SETS - 1][b][u] = __builtin_fmaf(p[i * QB + b], w, word_sum[SETS - 1][b][u]);
                  }
            }
          } else {
          for (int mc = 0; mc < L.mc; ++mc) {
            const int m = mc * 64 + hm;
            if (m >= L.mh) break;
            const uint8_t* cb = ct + (h0 + m) / 2 * kCodeRun;
            const int sh = ((h0 + m) & 1) * 4;
            float* hc = hist + mc * 1024 + lane;
            for (int j = j0; j < j1; j += 8) {
              u32x2 c8 = *reinterpret_cast<const u32x2*>(cb + j);
              c8 >>= sh;
              float p[8 * QB], p2[8 * QB];
              load_weights<8 * QB>(pr + j * QB, p);
              if (GRAD) load_weights<8 * QB>(pr2 + j * QB, p2);
#pragma unroll
              for (int i = 0; i < 8; i += 2) {
                const u32 ca = (c8[i >> 2] >> (8 * (i & 3))) & 15u, cc = (c8[i >> 2] >> (8 * (i & 3) + 8)) & 15u;
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                  if (GRAD) add_pair(hc + b * L.mc * 1024, ca, cc, p2[i * QB + b], p2[(i + 1) * QB + b]);
                  add_pair(hc + ((SETS - 1) * QB + b) * L.mc * 1024, ca, cc, p[i * QB + b], p[(i + 1) * QB + b]);
                }
              }
            }
          }
          }
        }
      }
    }
    __syncthreads();
    for (int t = threadIdx.x; t < nout; t += 256) {
      float a[SETS][QB];
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        a[SETS - 1][b] = lds[L.cacc + ((SETS - 1) * QB + b) * nout + t];
        if (GRAD) a[0][b] = lds[L.cacc + b * nout + t];
      }
#pragma unroll 4
      for (int s = 0; s < nseg; ++s) {
        const float c = A.centroids[(int64_t)segs[s].list * d + hd0 + t];
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          a[SETS - 1][b] = __builtin_fmaf(lds[L.bias + s * QB + b], c, a[SETS - 1][b]);
          if (GRAD) a[0][b] = __builtin_fmaf(lds[L.bias2 + s * QB + b], c, a[0][b]);
        }
      }
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        lds[L.cacc + ((SETS - 1) * QB + b) * nout + t] = a[SETS - 1][b];
        if (GRAD) lds[L.cacc + b * nout + t] = a[0][b];
      }
    }
    if (next >= c_end) break;
  }
  // the wavefronts' and row groups' histograms become one: H[set][b][m][c], over the first of them
  __syncthreads();
  float* H = lds + (DS > 0 ? L.score : L.hist);
  if (DS > 0) {                                // (over the weights: [set][query][wavefront][lane][DS])
#pragma unroll
    for (int sb = 0; sb < SETS * QB; ++sb)
#pragma unroll
      for (int u = 0; u < (DS > 0 ? DS : 1); ++u)
        H[((sb * kWaves + wave) * 64 + lane) * DS + u] = hist_lane ? word_sum[sb / QB][sb % QB][u] : 0.f;
  } else
  for (int i = threadIdx.x; i < SETS * QB * L.mh * 16; i += 256) {
    const int c = i & 15, m = (i >> 4) % L.mh, sb = (i >> 4) / L.mh;
    const int mc = m >> 6, l0 = L.mh < 64 ? m : m & 63;
    float v = 0.f;
    for (int w = 0; w < kWaves; ++w)
      for (int r = 0; r < rstep; ++r) v += lds[L.hist + ((w * SETS * QB + sb) * L.mc + mc) * 1024 + c * 64 + l0 + r * L.mh];
    // (every sum reads its own cells; the first of them takes the result)
    H[(sb * L.mc + mc) * 1024 + c * 64 + l0] = v;
  }
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    sum[b] = wave_sum(sum[b]);
    sum2[b] = wave_sum(sum2[b]);
    if (lane == 0) { lds[L.red + wave * 2 * QB + b] = sum[b]; lds[L.red + wave * 2 * QB + QB + b] = sum2[b]; }
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < QB; ++b) {
    if (q0 + b >= A.nq) break;
    float* out = A.part + ((q0 + b) * A.nsplit + split) * A.ld;
    if (threadIdx.x == 0) {
      float s = 0.f, s2 = 0.f;
      for (int w = 0; w < kWaves; ++w) { s += lds[L.red + w * 2 * QB + b]; s2 += lds[L.red + w * 2 * QB + QB + b]; }
      out[0] = GRAD ? s2 : mx[b];
      out[1] = s;
      if (GRAD) out[2] = shift[b];
    }
    for (int i = threadIdx.x; i < SETS * nout; i += 256) {
      const int set = i / nout, t = i - set * nout, m = t / dsub, u = t - m * dsub;
      float v = lds[L.cacc + (set * QB + b) * nout + t];
      if (DS > 0) {
        for (int w = 0; w < kWaves; ++w)
          for (int r = 0; r < rstep; ++r) v += H[(((set * QB + b) * kWaves + w) * 64 + r * L.mh + m) * DS + u];
      } else {
        const float* cb = A.codebooks + (int64_t)(h0 + m) * 16 * dsub + u;
        const float* h = H + ((set * QB + b) * L.mc + (m >> 6)) * 1024 + (L.mh < 64 ? m : m & 63);
#pragma unroll
        for (int c = 0; c < 16; ++c) v = __builtin_fmaf(h[c * 64], cb[c * dsub], v);
      }
      out[(GRAD ? 3 : 2) + i] = v;
    }
  }
}


// ---- many queries over whole lists: decoded tiles on the matrix cores ------------------------------
// Queries of one call share their rows when all lists are read, and a row decoded once serves 16 or 64 of them: the
// operands of v_mfma_f32_16x16x32_f16 are put together in registers from codeword tables in LDS, nothing is decoded to
// memory.  A tile is 64 rows by 16 NQ queries:
//   scores  S^T = K q^T: a wavefront takes 16 rows (operand A: lane = row lane & 15, 8 components a step; a lane of group
//           g = lane >> 4 goes through the codes [g mq, (g + 1) mq) of its row, so its code bytes are consecutive; a
//           codeword is looked up in pieces of W components, {W heads, W tails}, padded to whole pieces),
//   weights p = e^(s - m) 2^14 in fp16 (fp32 queries: head and tail) through LDS, to lie along rows,
//   product O^T = V^T p^T: a wavefront takes 16 components of every 64 (operand A: lane = component, 8 rows a step,
//           looked up one by one in a table [component][16]).
// The centroid of a list adds a constant to its scores and sum(p) centroid to the product, both once per list and part.
// Every component has a power of two of its own, which brings its largest codeword to [2^14, 2^15), the top of fp16's range:
// tables hold its codewords times that, queries its value over it (and times a power of two of the query that brings the
// largest of these there), results are taken back by it at the end.  So head and tail keep 2^-24 of a codeword or 2^-39 of its
// component's largest, whatever the sizes of other components, and scores are good to fp32; 16-bit queries are exact down to
// 2^-31 of the largest such value.  Weights keep 11 bits for 16-bit queries, whose results have no more, and 22 for fp32.
// The gradient's tile computes p from lse and the product of g with the values, w = p <g, t> and adds w k and p k; both
// relative to the centroid part of <g, v> of the present list, which is exchanged when the list changes.
// Bound by nothing alone: of a tile's time the score products, the weighted products, the staging of codes and the maxima
// take a fifth to a third each, and they meet at two barriers.  8 queries x 131,072 codes of 64 sub-quantizers, 128 and 128
// components: 31 us; 2048 x 16,384 under causal limits 110 us, the gradient of 1024 of them 118 us.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTileRows = 64;
constexpr int kTableBits = 14;                 // weights are held times 2^14

struct CodeSet {                               // sub-quantizers [m0, m0 + n) as rows of an operand
  int m0, n, mq, ppc, steps, stride, entry;    // codes of a lane group, pieces of a codeword, steps; bytes of a staged row, of a piece
};
__host__ __device__ inline CodeSet code_set(int m0, int n, int dsub, int w) {
  CodeSet c;
  const int per = 8 / w;
  c.m0 = m0; c.n = n;
  c.mq = ((n + 3) / 4 + per - 1) / per * per;
  c.ppc = (dsub + w - 1) / w;
  c.steps = c.ppc * c.mq / per;
  c.stride = 4 * c.mq + 4;
  c.entry = 4 * w;
  return c;
}
struct TileLds {                               // bytes
  int ktab, gtab, vtab, qf, gf, krow, grow, vcol, p, ids, red, stat, cent, exps, total;
  int p_stride, p_set, stage;
};
// 64-component runs of the result that a tile kernel is made for
__host__ __device__ inline int tile_runs(int nout) { return nout <= 64 ? 1 : (nout <= 128 ? 2 : (nout <= 256 ? 4 : 8)); }
__host__ __device__ inline TileLds tile_lds(const IvfpqDims& g, int dk, int v0, int w, int nq, int planes, bool grad) {
  TileLds o{};
  int at = 0;
  auto take = [&](int n) { const int b = at; at += (n + 15) / 16 * 16; return b; };
  const int dv = g.d - v0, mk = dk / g.dsub, mv = dv / g.dsub;
  const CodeSet k = code_set(0, mk, g.dsub, w), v = code_set(g.M - mv, mv, g.dsub, w);
  const int nout = grad ? dk : dv, mo = grad ? mk : mv;
  o.ktab = take(k.ppc * 4 * k.mq * 16 * k.entry);
  o.gtab = take(grad ? v.ppc * 4 * v.mq * 16 * v.entry : 0);
  o.vtab = take(tile_runs(nout) * 64 * 64);
  o.qf = take(planes * nq * k.steps * 1024);
  o.gf = take(grad ? planes * nq * v.steps * 1024 : 0);
  o.krow = take(kTileRows * k.stride);           // a stage: rows' codes, their ids; two of them
  o.grow = take(grad ? kTileRows * v.stride : 0);
  o.vcol = take(mo * 72);
  o.ids = take(kTileRows * 8);
  o.stage = at - o.krow;
  at += o.stage;
  o.p_stride = kTileRows * 2 + 16;
  o.p_set = planes * nq * 16 * o.p_stride;
  o.p = take((grad ? 2 : 1) * o.p_set);
  o.red = take(4 * 2 * nq * 16 * 4);
  o.stat = take(nq * 16 * 3 * 4);
  o.cent = take((dk + dv) * 4);
  o.exps = take((dk + dv) * 4);
  o.total = at;
  return o;
}

// A power of two p with p <= mx < 2 p (1 for 0)
__device__ __forceinline__ float power_below(float mx) {
  const int e = mx > 0.f && mx < __builtin_inff() ? (int)__builtin_amdgcn_frexp_expf(mx) - 1 : 0;
  return __builtin_ldexpf(1.f, e < -120 ? -120 : (e > 120 ? 120 : e));
}
__device__ __forceinline__ u32 pack_parts(float v) {     // {head, tail}
  const _Float16 hi = (_Float16)v, lo = (_Float16)(v - (float)hi);
  return (u32)__builtin_bit_cast(unsigned short, hi) | (u32)__builtin_bit_cast(unsigned short, lo) << 16;
}
// Four numbers as heads and tails, two to a word
__device__ __forceinline__ void pack_4(const float (&v)[4], u32 (&hi)[2], u32 (&lo)[2]) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f16x2 h = {(_Float16)v[2 * i], (_Float16)v[2 * i + 1]};
    const f16x2 l = {(_Float16)(v[2 * i] - (float)h[0]), (_Float16)(v[2 * i + 1] - (float)h[1])};
    hi[i] = __builtin_bit_cast(u32, h);
    lo[i] = __builtin_bit_cast(u32, l);
  }
}
// What pack_4 left of the four: heads, and tails too where PL is 2
template <int PL>
__device__ __forceinline__ void packed_4(const u32 (&hi)[2], const u32 (&lo)[2], float (&v)[4]) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (float)__builtin_bit_cast(f16x2, hi[i >> 1])[i & 1];
    if (PL == 2) v[i] += (float)__builtin_bit_cast(f16x2, lo[i >> 1])[i & 1];
  }
}
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Table of a code set: piece (j, code) of codeword c at ((j 4 mq + code) 16 + c) entry bytes, {W heads, W tails}, times 2 to
// the exponents of the set's components.
template <int W>
__device__ __forceinline__ void build_rows_table(char* tab, const CodeSet& c, const float* codebooks, int dsub, const int* exps) {
  const int n = c.ppc * 4 * c.mq * 16;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int w = i & 15, jc = i >> 4, code = jc % (4 * c.mq), j = jc / (4 * c.mq);
    _Float16* e = reinterpret_cast<_Float16*>(tab + i * c.entry);
#pragma unroll
    for (int t = 0; t < W; ++t) {
      const int u = j * W + t;
      const float v = code < c.n && u < dsub ? __builtin_ldexpf(codebooks[((int64_t)(c.m0 + code) * 16 + w) * dsub + u], exps[code * dsub + u]) : 0.f;
      const _Float16 hi = (_Float16)v;
      e[t] = hi;
      e[W + t] = (_Float16)(v - (float)hi);
    }
  }
}
// A vector's components under a lane group's codes [g mq, (g + 1) mq) of a set, handled by one thread: n of them from t0 on.
struct Share { int t0, n; };
__device__ __forceinline__ Share share_of(const CodeSet& c, int g, int dsub) {
  const int c0 = g * c.mq, c1 = c0 + c.mq < c.n ? c0 + c.mq : c.n;
  return {c0 * dsub, c1 > c0 ? (c1 - c0) * dsub : 0};
}
// f(t, value) for the share's components, eight loads in flight
template <int DT, typename F>
__device__ __forceinline__ void each_component(const void* row, const Share& s, F f) {
  int t = 0;
  for (; t + 8 <= s.n; t += 8) {
    float v[8];
    if (DT == VS_FP32) {
      __builtin_memcpy(v, static_cast<const float*>(row) + s.t0 + t, 32);
    } else if (DT == VS_FP16) {
      _Float16 e[8];
      __builtin_memcpy(e, static_cast<const _Float16*>(row) + s.t0 + t, 16);
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = (float)e[u];
    } else {
      __bf16 e[8];
      __builtin_memcpy(e, static_cast<const __bf16*>(row) + s.t0 + t, 16);
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = (float)e[u];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) f(t + u, v[u]);
  }
  for (; t < s.n; ++t) f(t, load_as_f32(row, s.t0 + t, DT));
}
template <typename F>
__device__ __forceinline__ void each_component(const void* row, const Share& s, int dtype, F f) {
  if (dtype == VS_FP32) each_component<VS_FP32>(row, s, f);
  else if (dtype == VS_FP16) each_component<VS_FP16>(row, s, f);
  else each_component<VS_BF16>(row, s, f);
}
__device__ __forceinline__ const void* row_of(const void* p, int64_t row, int ld, int dtype) {
  return static_cast<const char*>(p) + row * ld * (dtype == VS_FP32 ? 4 : 2);
}
// Operand B of a code set, [plane][block of 16][step][64 lanes]: the lane of query ql and group g holds its share in the
// order of the steps, times 2 to e less its component's exponent.  (The fragments hold zeros before.)
template <int W, int PL>
__device__ __forceinline__ void put_query_fragments(char* out, const CodeSet& c, int nqb, int ql, int g, const void* row,
                                                    int dtype, int dsub, const int* exps, int e) {
  constexpr int PER = 8 / W;
  const int plane = nqb * c.steps * 1024, per_j = c.mq / PER;
  char* lane_at = out + ((ql >> 4) * c.steps * 64 + g * 16 + (ql & 15)) * 16;
  int code = 0, u = 0;                         // of the component that comes next
  const Share sh = share_of(c, g, dsub);
  each_component(row, sh, dtype, [&](int i, float x) {
    const float v = __builtin_ldexpf(x, e - exps[sh.t0 + i]);
    const _Float16 hi = (_Float16)v;
    const int step = u / W * per_j + code / PER, t = code % PER * W + u % W;
    _Float16* at = reinterpret_cast<_Float16*>(lane_at + step * 1024) + t;
    at[0] = hi;
    if (PL == 2) at[plane / 2] = (_Float16)(v - (float)hi);
    if (++u == dsub) { u = 0; ++code; }
  });
}

// acc[qb] += rows (16 of this wavefront) x queries over a code set; acc's lane: query lane & 15, rows 4 (lane >> 4) + r
template <int W, int NQ, int PL>
__device__ __forceinline__ void rows_product(const char* tab, const CodeSet& c, const char* rows, const char* frag, f32x4 (&acc)[NQ]) {
  constexpr int PER = 8 / W;
  const int lane = lane_id(), g = lane >> 4;
  const char* mine = rows + (wave_id() * 16 + (lane & 15)) * c.stride + g * c.mq;
  const u32x4* b = reinterpret_cast<const u32x4*>(frag) + lane;
  const int n = NQ * c.steps * 64;
  const int per_j = c.mq / PER;
  for (int j = 0; j < c.ppc; ++j) {
    const char* t = tab + (j * 4 + g) * c.mq * 16 * c.entry;
    auto look = [&](int s, u32x4& hi, u32x4& lo) {
      u32 bytes;
      if (W == 4) bytes = *reinterpret_cast<const unsigned short*>(mine + s * 2);
      else bytes = *reinterpret_cast<const u32*>(mine + s * 4);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const char* e = t + (s * PER + i) * 16 * c.entry + ((bytes >> (8 * i)) & 15u) * c.entry;
        if (W == 4) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(e);
          hi[2 * i] = v[0]; hi[2 * i + 1] = v[1]; lo[2 * i] = v[2]; lo[2 * i + 1] = v[3];
        } else {
          const u32x2 v = *reinterpret_cast<const u32x2*>(e);
          hi[i] = v[0]; lo[i] = v[1];
        }
      }
    };
    auto multiply = [&](int s, const u32x4& hi, const u32x4& lo) {
      const int step = j * per_j + s;
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        const u32x4 q = b[(qb * c.steps + step) * 64];
        acc[qb] = mma(hi, q, acc[qb]);
        acc[qb] = mma(lo, q, acc[qb]);
        if (PL == 2) acc[qb] = mma(hi, b[n + (qb * c.steps + step) * 64], acc[qb]);
      }
    };
    int s = 0;
    for (; s + 4 <= per_j; s += 4) {              // four steps' look-ups in flight
      u32x4 hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) look(s + i, hi[i], lo[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) multiply(s + i, hi[i], lo[i]);
      settle_products();
    }
    for (; s < per_j; ++s) {
      u32x4 hi, lo;
      look(s, hi, lo);
      multiply(s, hi, lo);
      settle_products();
    }
  }
}

constexpr int SETS_OF(bool grad) { return grad ? 2 : 1; }
template <int W, int NQ, int NB, int PL, bool GRAD>
__global__ __launch_bounds__(256, SETS_OF(GRAD) * NQ * NB > 12 ? 1 : 2) void attend_tiles_kernel(ScanArgs A) {
  extern __shared__ __align__(16) char ldsb[];
  const TileLds L = tile_lds(A.g, A.dk, A.v0, W, NQ, PL, GRAD);
  constexpr int QT = NQ * 16, SETS = GRAD ? 2 : 1;
  const int lane = lane_id(), wave = wave_id(), g = lane >> 4, col = lane & 15;
  const int d = A.g.d, dsub = A.g.dsub, M = A.g.M, cs = A.g.code_size, dv = d - A.v0;
  const int mk = A.dk / dsub, mv = dv / dsub, mv0 = M - mv;
  const CodeSet K = code_set(0, mk, dsub, W), V = code_set(mv0, mv, dsub, W);
  const int nout = GRAD ? A.dk : dv, om0 = GRAD ? 0 : mv0, mo = GRAD ? mk : mv;
  const u32 wg = (u32)group_id();                              // (below 2^31)
  const int split = wg % A.nsplit;
  const int64_t q0 = (int64_t)(wg / A.nsplit) * QT;
  if (q0 >= A.nq) return;
  const int64_t r0 = split * A.per, r1 = r0 + A.per < A.ntotal ? r0 + A.per : A.ntotal;
  float* red = reinterpret_cast<float*>(ldsb + L.red);
  float* stat = reinterpret_cast<float*>(ldsb + L.stat);     // per query: factor of its products, of those of g; bound of w
  float* cent = reinterpret_cast<float*>(ldsb + L.cent);     // centroid of the list: [dk] keys, [dv] values

  // exponents of the key and value components (zeros take the largest one), then factors of every query
  int* kexp = reinterpret_cast<int*>(ldsb + L.exps);
  int* vexp = kexp + A.dk;
  constexpr int kNone = 1 << 20;
  int kmin = kNone, vmin = kNone;
  for (int t = threadIdx.x; t < A.dk + dv; t += 256) {
    const int comp = t < A.dk ? t : A.v0 + t - A.dk, m = comp / dsub;
    const float* cb = A.codebooks + (int64_t)m * 16 * dsub + (comp - m * dsub);
    float mx = 0.f;
#pragma unroll
    for (int c = 0; c < 16; ++c) mx = fmaxf(mx, fabsf(cb[c * dsub]));
    const int e = mx > 0.f ? top_exponent(mx) : kNone;
    kexp[t] = e;
    if (t < A.dk) kmin = e < kmin ? e : kmin;
    else vmin = e < vmin ? e : vmin;
  }
  for (int i = threadIdx.x; i < PL * NQ * K.steps * 64; i += 256) reinterpret_cast<u32x4*>(ldsb + L.qf)[i] = u32x4{0, 0, 0, 0};
  if (GRAD)
    for (int i = threadIdx.x; i < PL * NQ * V.steps * 64; i += 256) reinterpret_cast<u32x4*>(ldsb + L.gf)[i] = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) {
    const int a = __shfl_xor(kmin, w), b = __shfl_xor(vmin, w);
    kmin = a < kmin ? a : kmin;
    vmin = b < vmin ? b : vmin;
  }
  if (lane == 0) { reinterpret_cast<int*>(red)[wave] = kmin; reinterpret_cast<int*>(red)[4 + wave] = vmin; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int a = reinterpret_cast<int*>(red)[w], b = reinterpret_cast<int*>(red)[4 + w];
    kmin = a < kmin ? a : kmin;
    vmin = b < vmin ? b : vmin;
  }
  // No more than 24 above the smallest: sums hold centroids as well, times the same power, and 24 more bits of range are what
  // parts of smaller components have anyway.
  for (int t = threadIdx.x; t < A.dk + dv; t += 256) {
    const int low = t < A.dk ? kmin : vmin, most = (low == kNone ? 0 : low) + 24;
    kexp[t] = kexp[t] < most ? kexp[t] : most;
  }
  __syncthreads();
  // four threads a query, a lane group's share of the components each
  const int ql = threadIdx.x >> 2, qg = threadIdx.x & 3;
  const bool q_thread = ql < QT;
  const void* q_row = q_thread && q0 + ql < A.nq ? row_of(A.q, q0 + ql, A.dk, A.dtype) : nullptr;
  const void* g_row = GRAD && q_row ? row_of(A.g_out, q0 + ql, dv, A.dtype) : nullptr;
  if (q_thread) {
    float mx = 0.f, gx = 0.f, g1 = 0.f;
    const Share ks = share_of(K, qg, dsub), vs = share_of(V, qg, dsub);
    if (q_row) each_component(q_row, ks, A.dtype, [&](int i, float v) { mx = fmaxf(mx, __builtin_ldexpf(fabsf(v), -kexp[ks.t0 + i])); });
    if (g_row)
      each_component(g_row, vs, A.dtype, [&](int i, float v) {
        const float w = __builtin_ldexpf(fabsf(v), -vexp[vs.t0 + i]);
        gx = fmaxf(gx, w);
        g1 += w;
      });
#pragma unroll
    for (int w = 1; w < 4; w <<= 1) {
      mx = fmaxf(mx, __shfl_xor(mx, w));
      if (GRAD) { gx = fmaxf(gx, __shfl_xor(gx, w)); g1 += __shfl_xor(g1, w); }
    }
    const int e = top_exponent(mx);
    if (qg == 0) stat[ql] = __builtin_ldexpf(1.f, -e);
    if (q_row) put_query_fragments<W, PL>(ldsb + L.qf, K, NQ, ql, qg, q_row, A.dtype, dsub, kexp, e);
    if (GRAD) {
      const int ge = top_exponent(gx);
      // |<g, t>| <= sum |g_t| max |t|, below twice the last one
      if (qg == 0) { stat[QT + ql] = __builtin_ldexpf(1.f, -ge); stat[2 * QT + ql] = power_below(g1 * 32768.f); }
      if (g_row) put_query_fragments<W, PL>(ldsb + L.gf, V, NQ, ql, qg, g_row, A.dtype, dsub, vexp, ge);
    }
  }
  __syncthreads();
  build_rows_table<W>(ldsb + L.ktab, K, A.codebooks, dsub, kexp);
  if (GRAD) build_rows_table<W>(ldsb + L.gtab, V, A.codebooks, dsub, vexp);
  const int* oexp = GRAD ? kexp : vexp;                      // of the results' components
  for (int i = threadIdx.x; i < NB * 64 * 16; i += 256) {
    const int t = i >> 4, c = i & 15, m = t / dsub;
    reinterpret_cast<u32*>(ldsb + L.vtab)[i] = t < nout ? pack_parts(__builtin_ldexpf(A.codebooks[((int64_t)(om0 + m) * 16 + c) * dsub + t - m * dsub], oexp[t])) : 0u;
  }
  __syncthreads();

  int64_t limit[NQ], seen_to = INT64_MIN;
  bool all_in = true;                                        // no query that sees nothing (past the last one, say)
  float fs[NQ], fg[NQ], fw[NQ], lse[NQ], bias[NQ], mx[NQ], lp[NQ], lw[NQ], sum[NQ], sum2[NQ];
  f32x4 o[SETS][NB][NQ] = {};
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int64_t qi = q0 + qb * 16 + col;
    const bool in = qi < A.nq;
    limit[qb] = !in ? INT64_MIN : (A.limits ? A.limits[qi] : INT64_MAX);
    lse[qb] = GRAD && in ? A.lse[qi] * kLog2e : 0.f;
    if (GRAD && lse[qb] == neg_inf()) limit[qb] = INT64_MIN;
    all_in = all_in && limit[qb] != INT64_MIN;
    fs[qb] = A.scale * stat[qb * 16 + col] * kLog2e;         // (scores in units of log 2 inside)
    fg[qb] = GRAD ? stat[QT + qb * 16 + col] : 0.f;
    fw[qb] = GRAD ? 1.f / stat[2 * QT + qb * 16 + col] : 0.f;
    mx[qb] = neg_inf(); lp[qb] = 0.f; lw[qb] = 0.f; sum[qb] = 0.f; sum2[qb] = 0.f; bias[qb] = 0.f;
    seen_to = limit[qb] > seen_to ? limit[qb] : seen_to;
  }
#pragma unroll
  for (int w = 1; w < 16; w <<= 1) { const int64_t t = __shfl_xor(seen_to, w); seen_to = t > seen_to ? t : seen_to; }
  int vdim[NB];                                              // this lane's components' columns of staged codes
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int t = (nb * 4 + wave) * 16 + col;
    vdim[nb] = (t < nout ? t : nout - 1) / dsub * 72;
  }

  // sums over the list that ends: centroid parts of the results, and (gradient) the exchange of <g, centroid>
  float gbias[NQ], shift[NQ];
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) { gbias[qb] = 0.f; shift[qb] = 0.f; }
  int list = -1;
  auto close_list = [&]() {
    if (list < 0) return;
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      float p = lp[qb], w = lw[qb];
      p += __shfl_xor(p, 16); p += __shfl_xor(p, 32);
      if (GRAD) { w += __shfl_xor(w, 16); w += __shfl_xor(w, 32); }
      if (g == 0) { red[(wave * 2) * QT + qb * 16 + col] = p; if (GRAD) red[(wave * 2 + 1) * QT + qb * 16 + col] = w; }
      lp[qb] = 0.f; lw[qb] = 0.f;
    }
    __syncthreads();
    const float* c = GRAD ? cent : cent + A.dk;
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      float p = 0.f, w = 0.f;
#pragma unroll
      for (int v = 0; v < 4; ++v) { p += red[(v * 2) * QT + qb * 16 + col]; if (GRAD) w += red[(v * 2 + 1) * QT + qb * 16 + col]; }
      sum[qb] += p;                              // (sums times 2^14; o also times its component's power; lw and o of w over its bound)
      if (GRAD) sum2[qb] = __builtin_fmaf(w, stat[2 * QT + qb * 16 + col], sum2[qb]);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = (nb * 4 + wave) * 16 + 4 * g + r;
          const float cv = t < nout ? __builtin_ldexpf(c[t], oexp[t]) : 0.f;
          o[SETS - 1][nb][qb][r] = __builtin_fmaf(cv, p, o[SETS - 1][nb][qb][r]);
          if (GRAD) o[0][nb][qb][r] = __builtin_fmaf(cv, w, o[0][nb][qb][r]);
        }
    }
    __syncthreads();
  };
  auto open_list = [&](int l) {
    list = l;
    const float* c = A.centroids + (int64_t)l * d;
    for (int t = threadIdx.x; t < A.dk; t += 256) cent[t] = c[t];
    for (int t = threadIdx.x; t < dv; t += 256) cent[A.dk + t] = c[A.v0 + t];
    __syncthreads();
    if (q_thread) {                                          // <q, c>, <g, c> in fp32
      float s = 0.f, s2 = 0.f;
      const Share ks = share_of(K, qg, dsub), vs = share_of(V, qg, dsub);
      if (q_row) each_component(q_row, ks, A.dtype, [&](int t, float v) { s = __builtin_fmaf(v, cent[ks.t0 + t], s); });
      if (g_row) each_component(g_row, vs, A.dtype, [&](int t, float v) { s2 = __builtin_fmaf(v, cent[A.dk + vs.t0 + t], s2); });
#pragma unroll
      for (int w = 1; w < 4; w <<= 1) { s += __shfl_xor(s, w); if (GRAD) s2 += __shfl_xor(s2, w); }
      if (qg == 0) { red[ql] = s * A.scale * kLog2e; red[QT + ql] = s2; }
    }
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      bias[qb] = red[qb * 16 + col];
      if (GRAD) {                                            // sums relative to the new list's <g, c>
        const float now = red[QT + qb * 16 + col], by = gbias[qb] - now;
        sum2[qb] = __builtin_fmaf(by, sum[qb], sum2[qb]);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[0][nb][qb][r] = __builtin_fmaf(by * fw[qb], o[1][nb][qb][r], o[0][nb][qb][r]);
        gbias[qb] = now;
      }
    }
    __syncthreads();
  };

  // a tile's codes and ids, one tile ahead in registers: thread = row lane, words wave, wave + 4, ..
  constexpr int kWords = 4;
  const int words = (cs + 3) / 4;
  u32 ahead[kWords];
  int64_t ahead_id = 0;
  auto fetch = [&](int64_t pos, int n) {
    const uint8_t* row = A.codes + (pos + (lane < n ? lane : 0)) * cs;
    // (a word that the row does not fill is loaded so that it ends with the row, and shifted where it is used: no load
    // hangs on a condition, so none is waited for)
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int w = wave + 4 * i;
      if (w < words) {
        if (cs >= 4) __builtin_memcpy(&ahead[i], row + (4 * w + 4 <= cs ? 4 * w : cs - 4), 4);
        else ahead[i] = code_word(row, w, cs);
      }
    }
    if (A.limits) ahead_id = lane < n ? A.ids[pos + lane] : INT64_MAX;
  };

  int64_t pos = r0;
  int cur = -1;
  int64_t cur_end = r0;
  auto advance = [&]() {                                      // list and end of the run that pos lies in
    if (pos < r1 && pos >= cur_end) {
      cur = cur < 0 ? list_of_position(A.list_off, A.g.nlist, pos) : cur + 1;
      while (A.list_off[cur + 1] <= pos) ++cur;
      cur_end = A.list_off[cur + 1] < r1 ? A.list_off[cur + 1] : r1;
    }
  };
  // The next run that some query sees, its codes in registers: {rows, list}; rows 0 at the end.
  int next_n = 0, next_list = -1;
  auto take_next = [&]() {
    while (true) {
      advance();
      next_n = pos < r1 ? (int)(cur_end - pos < kTileRows ? cur_end - pos : kTileRows) : 0;
      if (next_n == 0) return;
      next_list = cur;
      fetch(pos, next_n);
      pos += next_n;
      if (!A.limits || __ballot(ahead_id < seen_to) != 0) return;   // (the same rows in every wavefront)
    }
  };
  // Codes as bytes: along rows for the scores, along components for the product.
  auto put_stage = [&](int which) {
    char* st = ldsb + which * L.stage;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const int w = wave + 4 * i;
      if (w < words) {
        const u32 word = ahead[i] >> (cs >= 4 && 4 * w + 4 > cs ? 8 * (4 * w + 4 - cs) : 0);
        const u32 even = word & 0x0F0F0F0Fu, odd = (word >> 4) & 0x0F0F0F0Fu;
        const u32 b0 = __builtin_amdgcn_perm(odd, even, 0x05010400u), b1 = __builtin_amdgcn_perm(odd, even, 0x07030602u);
        const int m = w * 8;
        auto row_bytes = [&](char* rows, const CodeSet& c) {
          const int at = m - c.m0;
          char* out = rows + lane * c.stride;
          if (at >= 0 && at + 8 <= 4 * c.mq && (at & 3) == 0) {
            *reinterpret_cast<u32*>(out + at) = b0;
            *reinterpret_cast<u32*>(out + at + 4) = b1;
          } else if (at + 8 > 0 && at < 4 * c.mq) {
#pragma unroll
            for (int u = 0; u < 8; ++u)
              if (at + u >= 0 && at + u < 4 * c.mq) out[at + u] = (char)((u < 4 ? b0 : b1) >> (8 * (u & 3)));
          }
        };
        row_bytes(st + L.krow, K);
        if (GRAD) row_bytes(st + L.grow, V);
        char* cols = st + L.vcol + (m - om0) * 72 + lane;
        if (m >= om0 && m + 8 <= om0 + mo) {
#pragma unroll
          for (int u = 0; u < 8; ++u) cols[u * 72] = (char)((u < 4 ? b0 : b1) >> (8 * (u & 3)));
        } else {
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (m + u >= om0 && m + u < om0 + mo) cols[u * 72] = (char)((u < 4 ? b0 : b1) >> (8 * (u & 3)));
        }
      }
    }
    if (wave == 0 && A.limits) reinterpret_cast<int64_t*>(st + L.ids)[lane] = ahead_id;
  };

  take_next();
  int here = next_n, here_list = next_list, turn = 0;
  if (here > 0) {
    put_stage(0);
    take_next();
  }
  block_sync_lds();
  // A stage is written while the one before it is multiplied: two barriers a tile, after the maxima and after the weights,
  // which leave the codes that are on their way alone.
  while (here > 0) {
    if (here_list != list) { close_list(); open_list(here_list); }
    char* st = ldsb + (turn & 1) * L.stage;
    const int64_t* ids = reinterpret_cast<const int64_t*>(st + L.ids);
    f32x4 s[NQ] = {}, t[NQ] = {};
    rows_product<W, NQ, PL>(ldsb + L.ktab, K, st + L.krow, ldsb + L.qf, s);
    if (GRAD) rows_product<W, NQ, PL>(ldsb + L.gtab, V, st + L.grow, ldsb + L.gf, t);
    const int row = wave * 16 + 4 * g;
    // which of the 4 x NQ pairs count: all of a whole run that every query sees to its end
    u32 sees = ~0u;
    if (here < kTileRows || A.limits || !all_in) {
      sees = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t id = A.limits ? ids[row + r] : 0;
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) sees |= (u32)(row + r < here && id < limit[qb]) << (qb * 4 + r);
      }
    }
    if (GRAD) {
      block_sync_lds();                                        // the weights of the tile before have been multiplied
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[qb][r] = __builtin_fmaf(s[qb][r], fs[qb], bias[qb]);
    } else {
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        float m = neg_inf();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float v = __builtin_fmaf(s[qb][r], fs[qb], bias[qb]);
          s[qb][r] = (sees >> (qb * 4 + r)) & 1u ? v : neg_inf();
          m = fmaxf(m, s[qb][r]);
        }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        if (g == 0) red[wave * QT + qb * 16 + col] = m;
      }
      block_sync_lds();
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        float m = mx[qb];
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, red[v * QT + qb * 16 + col]);
        if (__ballot(m > mx[qb]) != 0) {
          const float f = mx[qb] == neg_inf() ? 1.f : __builtin_amdgcn_exp2f(mx[qb] - m);      // (nothing yet: zeros to scale)
          lp[qb] *= f;
          sum[qb] *= f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) o[0][nb][qb] *= f;
          mx[qb] = m;
        }
      }
    }
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      // weights times 2^14 throughout
      const float base = (GRAD ? lse[qb] : (mx[qb] > neg_inf() ? mx[qb] : 0.f)) - (float)kTableBits;
      float p[4], w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = __builtin_amdgcn_exp2f(s[qb][r] - base);
        w[r] = 0.f;
        if (GRAD) {
          if (!((sees >> (qb * 4 + r)) & 1u)) p[r] = 0.f;
          w[r] = p[r] * (t[qb][r] * fg[qb]);
          if (!((sees >> (qb * 4 + r)) & 1u)) w[r] = 0.f;
          w[r] *= fw[qb];
        } else {
          lp[qb] += p[r];
        }
      }
      u32 ph[2], pl[2], wh[2], wl[2];
      pack_4(p, ph, pl);
      if (GRAD) {
        // Summed as they are multiplied: sum w k and (sum w / sum p) sum p k nearly cancel where few rows have any weight, and
        // the roundings of the weights must do so with them.
        pack_4(w, wh, wl);
        float pk[4], wk[4];
        packed_4<PL>(ph, pl, pk);
        packed_4<PL>(wh, wl, wk);
#pragma unroll
        for (int r = 0; r < 4; ++r) { lp[qb] += pk[r]; lw[qb] += wk[r]; }
      }
      char* out = ldsb + L.p + (SETS - 1) * L.p_set + (qb * 16 + col) * L.p_stride + row * 2;
      *reinterpret_cast<u32x2*>(out) = u32x2{ph[0], ph[1]};
      if (PL == 2) *reinterpret_cast<u32x2*>(out + QT * L.p_stride) = u32x2{pl[0], pl[1]};
      if (GRAD) {
        out -= L.p_set;
        *reinterpret_cast<u32x2*>(out) = u32x2{wh[0], wh[1]};
        if (PL == 2) *reinterpret_cast<u32x2*>(out + QT * L.p_stride) = u32x2{wl[0], wl[1]};
      }
    }
    here = next_n;
    here_list = next_list;
    ++turn;
    if (here > 0) {
      put_stage(turn & 1);
      take_next();
    }
    block_sync_lds();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 b[SETS][PL][NQ];
#pragma unroll
      for (int st = 0; st < SETS; ++st)
#pragma unroll
        for (int pl = 0; pl < PL; ++pl)
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb)
            b[st][pl][qb] = *reinterpret_cast<const u32x4*>(ldsb + L.p + st * L.p_set + (pl * QT + qb * 16 + col) * L.p_stride + ks * 64 + g * 16);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int t0 = (nb * 4 + wave) * 16;
        if (NB <= 4 || t0 < nout) {                             // (tables reach over NB 64 components)
        const u32x2 c8 = *reinterpret_cast<const u32x2*>(st + L.vcol + vdim[nb] + ks * 32 + g * 8);
        const char* tab = ldsb + L.vtab + (t0 + col) * 64;
        u32 e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const u32 c = (c8[i >> 2] >> (8 * (i & 3))) & 15u;
          e[i] = *reinterpret_cast<const u32*>(tab + c * 4);
        }
        u32x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          hi[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x05040100u);
          lo[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x07060302u);
        }
#pragma unroll
        for (int st = 0; st < SETS; ++st)
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb) {
            o[st][nb][qb] = mma(hi, b[st][0][qb], o[st][nb][qb]);
            o[st][nb][qb] = mma(lo, b[st][0][qb], o[st][nb][qb]);
            if (PL == 2) o[st][nb][qb] = mma(hi, b[st][PL - 1][qb], o[st][nb][qb]);
          }
        }
      }
    }
    settle_products();
  }
  close_list();
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int64_t qi = q0 + qb * 16 + col;
    if (qi >= A.nq) continue;
    float* out = A.part + (qi * A.nsplit + split) * A.ld;
    if (wave == 0 && g == 0) {
      constexpr float one = 1.f / (float)(1 << kTableBits);
      out[0] = GRAD ? sum2[qb] * one : mx[qb] * kLn2;
      out[1] = sum[qb] * one;
      if (GRAD) out[2] = gbias[qb];
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = (nb * 4 + wave) * 16 + 4 * g + r;
        if (t >= nout) continue;
        const int e = -kTableBits - oexp[t];
        if (GRAD) {
          out[3 + t] = __builtin_ldexpf(o[0][nb][qb][r], e) * stat[2 * QT + qb * 16 + col];
          out[3 + nout + t] = __builtin_ldexpf(o[SETS - 1][nb][qb][r], e);
        } else {
          out[2 + t] = __builtin_ldexpf(o[0][nb][qb][r], e);
        }
      }
  }
}

// Parts joined under their common maximum (forward) or added (backward): a workgroup takes 64 results of a query.  The
// parts' factors come first, a part a thread; then four wavefronts go through the parts, eight loads in flight each.
constexpr int kMaxParts = 2048;
template <bool GRAD>
__global__ __launch_bounds__(256) void attend_join_kernel(const float* __restrict__ part, int64_t nq, int nsplit, int64_t ld, int nout,
                                                          const float* __restrict__ g_lse, float scale, int dtype,
                                                          void* __restrict__ out, float* __restrict__ out_lse) {
  __shared__ float factor[kMaxParts];
  __shared__ float red[8];
  __shared__ float sums[4][64];
  const int64_t qi = blockIdx.x + (int64_t)gridDim.x * blockIdx.z;
  if (qi >= nq) return;
  const int lane = lane_id(), wave = wave_id(), t = blockIdx.y * 64 + lane;
  const float* p = part + qi * nsplit * ld;
  float inv = 1.f;
  bool nothing = false;                           // (backward) no row's weight: zeros, whatever the query and its gradients hold
  if (!GRAD) {
    float m = neg_inf();
    for (int s = threadIdx.x; s < nsplit; s += 256) m = fmaxf(m, p[s * ld]);
    m = wave_max(m);
    if (lane == 0) red[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float l = 0.f;
    for (int s = threadIdx.x; s < nsplit; s += 256) {
      const float f = p[s * ld] == neg_inf() ? 0.f : exp_neg(p[s * ld] - m);
      factor[s] = f;
      l += f == 0.f && p[s * ld] == neg_inf() ? p[s * ld + 1] : p[s * ld + 1] * f;    // (0, or a NaN, of a part without maximum)
    }
    l = wave_sum(l);
    if (lane == 0) red[4 + wave] = l;
    __syncthreads();
    l = red[4] + red[5] + red[6] + red[7];
    inv = l == 0.f ? 0.f : 1.f / l;
    if (out_lse && blockIdx.y == 0 && threadIdx.x == 0) out_lse[qi] = l == 0.f ? neg_inf() : m + logf(l);
  } else {
    // sum p (dp - mean + g_lse) k, every part relative to its own shift of dp
    // (mean of dp under weights that sum to 1 up to the roundings of scores and lse: divided by their own sum, a common
    // factor of all weights leaves it as it is)
    float mean = 0.f, total = 0.f;
    for (int s = threadIdx.x; s < nsplit; s += 256) {
      mean += __builtin_fmaf(p[s * ld + 2], p[s * ld + 1], p[s * ld]);
      total += p[s * ld + 1];
    }
    mean = wave_sum(mean);
    total = wave_sum(total);
    if (lane == 0) { red[wave] = mean; red[4 + wave] = total; }
    __syncthreads();
    mean = red[0] + red[1] + red[2] + red[3];
    total = red[4] + red[5] + red[6] + red[7];
    nothing = total == 0.f;
    if (!nothing) mean /= total;
    const float gl = g_lse ? g_lse[qi] : 0.f;
    for (int s = threadIdx.x; s < nsplit; s += 256) factor[s] = p[s * ld + 2] - mean + gl;
    inv = scale;
    __syncthreads();
  }
  const int tt = t < nout ? t : nout - 1;
  const float* a = p + (GRAD ? 3 : 2) + tt;
  float v = 0.f;
  int s = wave;
  for (; s + 28 < nsplit; s += 32) {
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = a[(int64_t)(s + 4 * i) * ld];
      if (GRAD) y[i] = a[(int64_t)(s + 4 * i) * ld + nout];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (GRAD) v += __builtin_fmaf(factor[s + 4 * i], y[i], x[i]);
      else v = __builtin_fmaf(x[i], factor[s + 4 * i], v);
    }
  }
  for (; s < nsplit; s += 4) {
    const float x = a[(int64_t)s * ld];
    if (GRAD) v += __builtin_fmaf(factor[s], a[(int64_t)s * ld + nout], x);
    else v = __builtin_fmaf(x, factor[s], v);
  }
  sums[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && t < nout)
    store_as(out, qi * nout + t, dtype, nothing ? 0.f : (sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane]) * inv);
}

// q [nq, dk] of any type -> fp32 [nq, d] with zeros behind
__global__ __launch_bounds__(256) void attend_pad_kernel(const void* __restrict__ q, int64_t nq, int dk, int d, int dtype,
                                                         float* __restrict__ out) {
  const int64_t i = group_id() * 256 + threadIdx.x;
  if (i >= nq * d) return;
  const int64_t r = i / d;
  const int t = (int)(i - r * d);
  out[i] = t < dk ? load_as_f32(q, r * dk + t, dtype) : 0.f;
}

constexpr int kMaxLds = 160 * 1024;

// Which tile kernel serves a call, if any: p->tiles, nq16 (16-query blocks of a tile), nb (64-component runs of the result)
void tiles_plan(const IvfpqDims& g, int64_t ntotal, int64_t nq, int dk, int v0, int dtype, int nprobe, bool grad, AttendPlan* p) {
  p->tiles = false;
  const int nout = grad ? dk : g.d - v0, planes = dtype == VS_FP32 ? 2 : 1;
  if (nprobe > 0 || nq < 4 || g.code_size > 64 || nout > 512) return;
  // Tiles or the scan.  The scan's work is its look-ups, nq ntotal (dk + d - v0) / dsub; a tile reads a code once for 16 or
  // 64 queries, but assembles operands for as many, begins later, and fills up a list's last 64 rows.  Scan and tiles in us,
  // fp16, dk = d = 128, M = 32 (millions of look-ups in brackets): 3000 codes, 64 queries (12) 26 and 39, 256 (49) 37 and 39,
  // 1024 (197) 87 and 42; 20,000, 8 queries (10) 26 and 27, 16 (20) 31 and 27, 64 (82) 47 and 38; 1,500,000, 2 queries (192)
  // 94 and 163, 4 (384) 148 and 158, 8 (768) 213 and 158; 20,000 in lists of 312, 64 queries (82) 52 and 51, 512 197 and 69;
  // in lists of 78, 64 queries 65 and 67, 512 252 and 91; in lists of 31, 64 queries 96 and 112, 512 366 and 142.  Results of
  // more than 256 components go 16 queries at a time: 50,000 codes of d = 320, M = 80, 8 queries (64) 62
  // and 55, 32 queries 205 and 104; sub-vectors of more than four components, which the scan takes as cheaply as short
  // ones: d = 384, M = 64, 32 queries (205) 89 and 117, 64 (410) 202 and 153; d = 768, M = 64, 256 queries 561 and 570.
  const double look_ups = (double)nq * (double)ntotal * (double)((dk + g.d - v0) / g.dsub), run = (double)ntotal / g.nlist;
  const double least = nout > 256 && g.dsub > 4 ? 256e6 : (nq > 16 || nout > 256 ? 48e6 : 16e6);
  if (run < 24. || look_ups < least * (1. + 100. / run)) return;
  p->w = g.dsub <= 2 ? 2 : 4;
  p->nb = tile_runs(nout);
  p->nq16 = nq > 16 && p->nb <= 4 ? (grad ? 2 : 4) : 1;   // (what a wavefront's registers hold)
  p->lds = tile_lds(g, dk, v0, p->w, p->nq16, planes, grad).total;
  if (p->nq16 > 1 && p->lds > kMaxLds) { p->nq16 = 1; p->lds = tile_lds(g, dk, v0, p->w, 1, planes, grad).total; }
  if (p->lds > kMaxLds) return;
  p->tiles = true;
  p->fits = true;
  p->qb = 16 * p->nq16;
  // Parts for three workgroups a CU.  Workgroups in all and us of a call: 2048 queries on 16,384 codes under causal limits 256
  // 175, 512 122, 768 118, 1024 140; one tile of 8 queries on 131,072 codes 256 42.4, 512 38.2, 768 38.1, 1024 38.2; on 524,288
  // 112, 75, 73 and 92; on 2,000,000 373, 226, 188 and 235; 300 queries (5 tiles) on 65,536 128, 135, 115 and 133.  One tile of
  // 64 queries, of which two fit a CU, on 524,288: 164, 114, 153 and 144; up to 131,072 codes the least part decides.
  const int64_t groups = (nq + p->qb - 1) / p->qb, want = (768 + groups - 1) / groups;
  const int64_t most = (ntotal + 255) / 256, splits = want < most ? want : most;
  p->per = ((ntotal + splits - 1) / splits + 63) / 64 * 64;
  p->nsplit = (int)((ntotal + p->per - 1) / p->per);
}

int scan_queries(const IvfpqDims& g, int dk, int v0, int64_t nq, bool probed, bool grad) {
  if (probed || nq == 1) return 1;
  return scan_lds(g, dk, v0, 2, grad).total * 4 <= kMaxLds / 2 ? 2 : 1;
}

}  // namespace

AttendPlan attend_plan(const IvfpqDims& g, int64_t ntotal, int64_t nq, int dk, int v0, int dtype, int nprobe, bool grad) {
  AttendPlan p{};
  p.nout = grad ? dk : g.d - v0;
  p.ld = grad ? 3 + 2 * (int64_t)p.nout : 2 + p.nout;
  tiles_plan(g, ntotal, nq, dk, v0, dtype, nprobe, grad, &p);
  if (p.tiles) return p;
  p.qb = scan_queries(g, dk, v0, nq, nprobe > 0, grad);
  p.lds = scan_lds(g, dk, v0, p.qb, grad).total * 4;
  p.fits = p.lds <= kMaxLds;
  // Parts of some 2048 rows, as many as make eight workgroups a CU: what a workgroup begins and ends with costs as much as
  // some 500 rows (333 queries of 3200 rows each: 2 parts 112 us, 3 125 us, 6 143 us; 1000 of 7800: 1 part 711 us, 2
  // 650 us, 3 618 us).  Few queries are cut finer, down to 256 rows, for two workgroups a CU.
  const int64_t groups = (nq + p.qb - 1) / p.qb > 0 ? (nq + p.qb - 1) / p.qb : 1;
  const int64_t rows = nprobe > 0 ? ntotal * nprobe / g.nlist : ntotal;
  const int64_t long_parts = std::min<int64_t>((2048 + groups - 1) / groups, (rows + 1024) / 2048);
  const int64_t short_parts = std::min<int64_t>((512 + groups - 1) / groups, (rows + 255) / 256);
  int64_t splits = long_parts > short_parts ? long_parts : short_parts;
  if (nprobe > 0 && splits > nprobe) splits = nprobe;
  if (splits < 1) splits = 1;
  if (nprobe > 0) {
    p.per = (nprobe + splits - 1) / splits;
    p.nsplit = (int)((nprobe + p.per - 1) / p.per);
  } else {
    p.per = ((ntotal + splits - 1) / splits + 63) / 64 * 64;
    if (p.per < 64) p.per = 64;
    p.nsplit = ntotal > 0 ? (int)((ntotal + p.per - 1) / p.per) : 1;
  }
  return p;
}

void launch_attend_pad(const void* q, int64_t nq, int dk, int d, int dtype, float* out, hipStream_t st) {
  attend_pad_kernel<<<grid_2d((nq * d + 255) / 256), 256, 0, st>>>(q, nq, dk, d, dtype, out);
}

void launch_attend(const AttendCall& c, const AttendPlan& p, bool grad, float* part, hipStream_t st) {
  const IvfStore& s = *c.ix;
  ScanArgs a{s.g, s.centroids, s.codebooks, s.codes, s.ids, s.list_off, s.ntotal, c.q, c.nq, c.dk, c.v0, c.dtype, c.scale,
             c.limits, c.probes, c.nprobe, p.nsplit, p.per, c.lse, c.g_out, part, p.ld};
  const dim3 g = grid_2d((c.nq + p.qb - 1) / p.qb * p.nsplit);
  auto run = [&](auto kern) {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLds);
    kern<<<g, 256, p.lds, st>>>(a);
  };
  if (p.tiles) {
#define TILES(W, NQ, NB)                                                        \
  do {                                                                          \
    constexpr int NG = NQ == 4 ? 2 : 1;                                         \
    if (c.dtype == VS_FP32) { if (grad) run(attend_tiles_kernel<W, NG, NB, 2, true>); else run(attend_tiles_kernel<W, NQ, NB, 2, false>); } \
    else { if (grad) run(attend_tiles_kernel<W, NG, NB, 1, true>); else run(attend_tiles_kernel<W, NQ, NB, 1, false>); } \
  } while (0)
#define TILES_W(W)                                                              \
  do {                                                                          \
    if (p.nq16 > 1) { if (p.nb == 1) TILES(W, 4, 1); else if (p.nb == 2) TILES(W, 4, 2); else TILES(W, 4, 4); } \
    else if (p.nb == 1) TILES(W, 1, 1);                                          \
    else if (p.nb == 2) TILES(W, 1, 2);                                          \
    else if (p.nb == 4) TILES(W, 1, 4);                                          \
    else TILES(W, 1, 8);                                                        \
  } while (0)
    if (p.w == 2) TILES_W(2);
    else TILES_W(4);
#undef TILES_W
#undef TILES
  } else {
#define SCAN(DS)                                                                                                \
  do {                                                                                                          \
    if (grad) { if (p.qb == 2) run(attend_scan_kernel<2, true, DS>); else run(attend_scan_kernel<1, true, DS>); } \
    else { if (p.qb == 2) run(attend_scan_kernel<2, false, DS>); else run(attend_scan_kernel<1, false, DS>); }    \
  } while (0)
    switch (scan_words(s.g, c.dk, c.v0, grad)) {
      case 4: SCAN(4); break;
      case 2: SCAN(2); break;
      case 1: SCAN(1); break;
      default: SCAN(0);
    }
#undef SCAN
  }
  const dim3 gq = grid_2d(c.nq), gj(gq.x, (unsigned)((p.nout + 63) / 64), gq.y);
  if (grad) attend_join_kernel<true><<<gj, 256, 0, st>>>(part, c.nq, p.nsplit, p.ld, p.nout, c.g_lse, c.scale, c.dtype, c.out, nullptr);
  else attend_join_kernel<false><<<gj, 256, 0, st>>>(part, c.nq, p.nsplit, p.ld, p.nout, nullptr, c.scale, c.dtype, c.out, c.out_lse);
}
