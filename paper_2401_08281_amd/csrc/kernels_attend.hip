// Attention over the vectors of a 4-bit IVF-PQ index, and its gradient for the queries.
//
// Both products of attention are taken in the code domain.  With keys and values x'_j = c_l + concat_m T_m[code_jm]:
//   s_ij  = scale <q, c_l> + sum_m LUT_m[code_jm],  LUT_m[c] = scale <q_m, T_m[c]>            (a look-up per sub-quantizer)
//   out_i = sum_l P_l c_l + concat_m sum_c H_m[c] T_m[c],  H_m[c] = sum of p_j with code_jm = c  (an addition per one)
// so a stored vector costs 2 M operations on LDS a query instead of 2 d products, whatever its dimension.
//
// A workgroup takes QB queries and a part of the rows, in rounds of up to 1024 rows: scores (one row a lane, all
// queries), their maximum, weights, then the histograms H (one sub-quantizer a lane).  A lane adds to its own column of
// its wavefront's H only: additions keep their order, banks never collide.  Partial results of the parts are joined by a
// second kernel.  Bound by LDS: one look-up of QB values and one addition per query for every code.
#include "../../include/vs_softmax.h"
#include "common.hpp"
#include "softmax.hpp"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kRound = 1024;        // rows of a round
constexpr int kSegments = 64;       // lists it may span
constexpr int kWaves = 4;
__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float exp_neg(float t) { return __builtin_amdgcn_exp2f(t * kLog2e); }
typedef __attribute__((address_space(3))) float* lds_float;
__device__ __forceinline__ void lds_add(float* p, float v) {
  __builtin_amdgcn_ds_faddf((lds_float)p, v, 0, 0, false);
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) v += __shfl_xor(v, w);
  return v;
}
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

struct Segment { int64_t pos; int32_t list, first, len, pad; };   // rows [first, first + len) of a round

// What a workgroup of QB queries keeps in LDS, in floats.
struct ScanLds {
  int lut, lut2, q, g, score, score2, hist, cacc, codes, bias, bias2, red, seg, total;
  int code_words;                    // words of a staged code (odd: no two rows start in one bank)
  int mh, mc;                        // histogrammed sub-quantizers; 64-lane chunks of them
};
__host__ __device__ inline ScanLds scan_lds(const IvfpqDims& g, int dk, int v0, int qb, bool grad) {
  ScanLds o{};
  const int mk = dk / g.dsub, mv = (g.d - v0) / g.dsub, out = grad ? dk : g.d - v0, sets = grad ? 2 : 1;
  o.mh = grad ? mk : mv;
  o.mc = (o.mh + 63) / 64;
  o.code_words = ((g.code_size + 3) / 4) | 1;
  int at = 0;
  auto take = [&](int n) { const int o2 = at; at += (n + 3) / 4 * 4; return o2; };
  o.lut = take(mk * 16 * qb);
  o.lut2 = take(grad ? mv * 16 * qb : 0);
  o.q = take(dk * qb);
  o.g = take(grad ? (g.d - v0) * qb : 0);
  o.score = take(kRound * qb);
  o.score2 = take(grad ? kRound * qb : 0);
  o.hist = take(kWaves * sets * qb * o.mc * 1024);
  o.cacc = take(sets * qb * out);
  o.codes = take(kWaves * 64 * o.code_words);
  o.bias = take(kSegments * qb);
  o.bias2 = take(grad ? kSegments * qb : 0);
  o.red = take(kWaves * 2 * qb + 8);
  o.seg = take((int)(sizeof(Segment) / 4) * kSegments + 8);
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
// Sum of the look-ups of sub-quantizers [m0, m1) of one row, in two chains: half the roundings in a row, and no addition
// waits for the one before.  The bias, usually the largest term, comes last.
template <int QB>
__device__ __forceinline__ void score_row(const uint8_t* row, int cs, int m0, int m1, const float* lut, const float* bias,
                                          float (&out)[QB]) {
  float acc[2][QB] = {};
  for (int w = m0 / 8; w * 8 < m1; ++w) {
    const u32 word = code_word(row, w, cs);
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
#pragma unroll
  for (int b = 0; b < QB; ++b) out[b] = (acc[0][b] + acc[1][b]) + bias[b];
}

template <int QB, bool GRAD>
__global__ __launch_bounds__(256) void attend_scan_kernel(ScanArgs A) {
  extern __shared__ __align__(16) float lds[];
  const ScanLds L = scan_lds(A.g, A.dk, A.v0, QB, GRAD);
  constexpr int SETS = GRAD ? 2 : 1;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const int d = A.g.d, dsub = A.g.dsub, M = A.g.M, cs = A.g.code_size, dv = d - A.v0;
  const int mk = A.dk / dsub, mv = dv / dsub, mv0 = M - mv;
  const int h0 = GRAD ? 0 : mv0, hd0 = GRAD ? 0 : A.v0, nout = GRAD ? A.dk : dv;   // the histogrammed sub-quantizers
  const int split = blockIdx.x % A.nsplit;
  const int64_t q0 = (int64_t)(blockIdx.x / A.nsplit) * QB;
  Segment* segs = reinterpret_cast<Segment*>(lds + L.seg);
  int* ctl = reinterpret_cast<int*>(lds + L.seg + (int)(sizeof(Segment) / 4) * kSegments);   // {segments, rows, next candidate}
  int64_t* offset = reinterpret_cast<int64_t*>(ctl + 4);         // rows of the next candidate that are done
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
  for (int i = threadIdx.x; i < kWaves * SETS * QB * L.mc * 1024; i += 256) lds[L.hist + i] = 0.f;
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
  const int rs = lane / (L.mh < 64 ? L.mh : 64), hm = lane % (L.mh < 64 ? L.mh : 64);
  const int rstep = L.mh < 64 ? 64 / L.mh : 1;
  const bool hist_lane = rs < rstep;

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
      int end = len0;                             // inclusive prefix sum
#pragma unroll
      for (int w = 1; w < 64; w <<= 1) {
        const int o = __shfl_up(end, w);
        if (lane >= w) end += o;
      }
      const int first = end - len0;
      const int len = first >= kRound ? 0 : (end > kRound ? kRound - first : len0);
      const u64 taken = __ballot(len > 0);
      if (len > 0) {
        const int at = __popcll(taken & ((1ull << lane) - 1));
        segs[at] = Segment{b, list, first, len, 0};
      }
      // the next round starts at the first candidate that is not used up
      const u64 open = __ballot(c < c_end && have > len);
      const int stop = open ? __ffsll(open) - 1 : 64;
      if (lane == (stop < 64 ? stop : 63)) {
        ctl[0] = __popcll(taken);
        ctl[1] = first + len < kRound ? first + len : kRound;
        ctl[2] = next + stop;
        *offset = stop < 64 ? (stop == 0 ? off + len : len) : 0;
      }
    }
    __syncthreads();
    const int nseg = ctl[0], rows = ctl[1], next = ctl[2];
    if (nseg == 0) {
      if (next >= c_end) break;
      continue;
    }
    // biases of the segments' lists
    for (int s = wave; s < nseg; s += kWaves) {
      const float* c = A.centroids + (int64_t)segs[s].list * d;
      float v[QB] = {}, v2[QB] = {};
      for (int t = lane; t < A.dk; t += 64)
#pragma unroll
        for (int b = 0; b < QB; ++b) v[b] = __builtin_fmaf(lds[L.q + b * A.dk + t], c[t], v[b]);
      if (GRAD)
        for (int t = lane; t < dv; t += 64)
#pragma unroll
          for (int b = 0; b < QB; ++b) v2[b] = __builtin_fmaf(lds[L.g + b * dv + t], c[A.v0 + t], v2[b]);
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
    int tile = 0;
    for (int s = 0; s < nseg; ++s) {
      const Segment sg = segs[s];
      for (int t0 = 0; t0 < sg.len; t0 += 64, ++tile) {
        if ((tile & (kWaves - 1)) != wave) continue;
        const int i = t0 + lane;
        if (i < sg.len) {
          const int64_t pos = sg.pos + i;
          const int64_t id = A.limits ? A.ids[pos] : 0;
          float acc[QB], acc2[QB];
          score_row<QB>(A.codes + pos * cs, cs, 0, mk, lds + L.lut, lds + L.bias + s * QB, acc);
          if (GRAD) score_row<QB>(A.codes + pos * cs, cs, mv0, M, lds + L.lut2, lds + L.bias2 + s * QB, acc2);
#pragma unroll
          for (int b = 0; b < QB; ++b) {
            const bool sees = id < limit[b];
            if (GRAD) {
              const float p = sees ? exp_neg(acc[b] - lse[b]) : 0.f;
              const float w = sees ? p * acc2[b] : 0.f;
              lds[L.score + (sg.first + i) * QB + b] = p;
              lds[L.score2 + (sg.first + i) * QB + b] = acc2[b];
              rp[b] += p;
              rw[b] += w;
            } else {
              const float v = sees ? acc[b] : neg_inf();
              lds[L.score + (sg.first + i) * QB + b] = v;
              top[b] = fmaxf(top[b], v);
            }
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
        for (int i = threadIdx.x; i < kWaves * QB * L.mc * 1024; i += 256) lds[L.hist + i] *= f[QB == 1 ? 0 : (i / (L.mc * 1024)) % QB];
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
    // histograms: a wavefront takes 64 rows, brings their codes into LDS, and adds row by row
    tile = 0;
    for (int s = 0; s < nseg; ++s) {
      const Segment sg = segs[s];
      for (int t0 = 0; t0 < sg.len; t0 += 64, ++tile) {
        if ((tile & (kWaves - 1)) != wave) continue;
        const int n = sg.len - t0 < 64 ? sg.len - t0 : 64;
        u32* ct = reinterpret_cast<u32*>(lds + L.codes) + wave * 64 * L.code_words;
        wave_lds_sync();
        if (lane < n) {
          const uint8_t* row = A.codes + (sg.pos + t0 + lane) * cs;
          for (int w = 0; w * 4 < cs; ++w) ct[lane * L.code_words + w] = code_word(row, w, cs);
        }
        wave_lds_sync();
        if (hist_lane) {
          const float* pr = lds + L.score + (sg.first + t0) * QB;
          const float* pr2 = lds + L.score2 + (sg.first + t0) * QB;
          for (int mc = 0; mc < L.mc; ++mc) {
            const int m = mc * 64 + hm;
            if (m >= L.mh) break;
            const uint8_t* cb = reinterpret_cast<const uint8_t*>(ct) + (h0 + m) / 2;
            const int sh = ((h0 + m) & 1) * 4;
            float* hc = hist + mc * 1024 + lane;
            for (int j = rs; j < n; j += rstep) {
              const int c = (cb[j * L.code_words * 4] >> sh) & 15;
#pragma unroll
              for (int b = 0; b < QB; ++b) {
                if (GRAD) {
                  lds_add(hc + (0 * QB + b) * L.mc * 1024 + c * 64, pr2[j * QB + b]);
                  lds_add(hc + (1 * QB + b) * L.mc * 1024 + c * 64, pr[j * QB + b]);
                } else {
                  lds_add(hc + b * L.mc * 1024 + c * 64, pr[j * QB + b]);
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
  float* H = lds + L.hist;
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
      const float* cb = A.codebooks + (int64_t)(h0 + m) * 16 * dsub + u;
      const float* h = H + ((set * QB + b) * L.mc + (m >> 6)) * 1024 + (L.mh < 64 ? m : m & 63);
      float v = lds[L.cacc + (set * QB + b) * nout + t];
#pragma unroll
      for (int c = 0; c < 16; ++c) v = __builtin_fmaf(h[c * 64], cb[c * dsub], v);
      out[(GRAD ? 3 : 2) + i] = v;
    }
  }
}

// One workgroup per query: parts joined under their common maximum (forward) or added (backward).
template <bool GRAD>
__global__ __launch_bounds__(256) void attend_join_kernel(const float* __restrict__ part, int nsplit, int64_t ld, int nout,
                                                          const float* __restrict__ g_lse, float scale, int dtype,
                                                          void* __restrict__ out, float* __restrict__ out_lse) {
  const int64_t qi = blockIdx.x;
  const float* p = part + qi * nsplit * ld;
  if (!GRAD) {
    float m = neg_inf();
    for (int s = 0; s < nsplit; ++s) m = fmaxf(m, p[s * ld]);
    float l = 0.f;
    for (int s = 0; s < nsplit; ++s) l += p[s * ld] == neg_inf() ? p[s * ld + 1] : p[s * ld + 1] * exp_neg(p[s * ld] - m);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int t = threadIdx.x; t < nout; t += 256) {
      float v = 0.f;
      for (int s = 0; s < nsplit; ++s)
        if (p[s * ld] != neg_inf()) v = __builtin_fmaf(p[s * ld + 2 + t], exp_neg(p[s * ld] - m), v);
      store_as(out, qi * nout + t, dtype, v * inv);
    }
    if (out_lse && threadIdx.x == 0) out_lse[qi] = l == 0.f ? neg_inf() : m + logf(l);
  } else {
    // sum p (dp - mean + g_lse) k, every part relative to its own shift of dp
    // (mean of dp under weights that sum to 1 up to the roundings of scores and lse: divided by their own sum, a common
    // factor of all weights leaves it as it is)
    float mean = 0.f, total = 0.f;
    for (int s = 0; s < nsplit; ++s) {
      mean += __builtin_fmaf(p[s * ld + 2], p[s * ld + 1], p[s * ld]);
      total += p[s * ld + 1];
    }
    if (total != 0.f) mean /= total;
    const float gl = g_lse ? g_lse[qi] : 0.f;
    for (int t = threadIdx.x; t < nout; t += 256) {
      float a = 0.f;
      for (int s = 0; s < nsplit; ++s)
        a += __builtin_fmaf(p[s * ld + 2] - mean + gl, p[s * ld + 3 + nout + t], p[s * ld + 3 + t]);
      store_as(out, qi * nout + t, dtype, scale * a);
    }
  }
}

// q [nq, dk] of any type -> fp32 [nq, d] with zeros behind
__global__ __launch_bounds__(256) void attend_pad_kernel(const void* __restrict__ q, int64_t nq, int dk, int d, int dtype,
                                                         float* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= nq * d) return;
  const int64_t r = i / d;
  const int t = (int)(i - r * d);
  out[i] = t < dk ? load_as_f32(q, r * dk + t, dtype) : 0.f;
}

constexpr int kMaxLds = 160 * 1024;

int scan_queries(const IvfpqDims& g, int dk, int v0, int64_t nq, bool probed, bool grad) {
  if (probed || nq == 1) return 1;
  return scan_lds(g, dk, v0, 2, grad).total * 4 <= kMaxLds / 2 ? 2 : 1;
}

}  // namespace

AttendPlan attend_plan(const IvfpqDims& g, int64_t ntotal, int64_t nq, int dk, int v0, int nprobe, bool grad) {
  AttendPlan p;
  p.nout = grad ? dk : g.d - v0;
  p.ld = grad ? 3 + 2 * (int64_t)p.nout : 2 + p.nout;
  p.qb = scan_queries(g, dk, v0, nq, nprobe > 0, grad);
  p.lds = scan_lds(g, dk, v0, p.qb, grad).total * 4;
  p.fits = p.lds <= kMaxLds;
  // some eight workgroups a CU; parts of 256 rows or one probe at least
  const int64_t groups = (nq + p.qb - 1) / p.qb, want = groups > 0 ? (2048 + groups - 1) / groups : 1;
  const int64_t most = nprobe > 0 ? nprobe : (ntotal + 255) / 256;
  int64_t splits = want < most ? want : most;
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
  attend_pad_kernel<<<(unsigned)((nq * d + 255) / 256), 256, 0, st>>>(q, nq, dk, d, dtype, out);
}

void launch_attend(const AttendCall& c, const AttendPlan& p, bool grad, float* part, hipStream_t st) {
  const IvfStore& s = *c.ix;
  ScanArgs a{s.g, s.centroids, s.codebooks, s.codes, s.ids, s.list_off, s.ntotal, c.q, c.nq, c.dk, c.v0, c.dtype, c.scale,
             c.limits, c.probes, c.nprobe, p.nsplit, p.per, c.lse, c.g_out, part, p.ld};
  const unsigned g = (unsigned)((c.nq + p.qb - 1) / p.qb * p.nsplit);
  auto run = [&](auto kern) {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLds);
    kern<<<g, 256, p.lds, st>>>(a);
  };
  if (grad) { if (p.qb == 2) run(attend_scan_kernel<2, true>); else run(attend_scan_kernel<1, true>); }
  else { if (p.qb == 2) run(attend_scan_kernel<2, false>); else run(attend_scan_kernel<1, false>); }
  if (grad) attend_join_kernel<true><<<(unsigned)c.nq, 256, 0, st>>>(part, p.nsplit, p.ld, p.nout, c.g_lse, c.scale, c.dtype, c.out, nullptr);
  else attend_join_kernel<false><<<(unsigned)c.nq, 256, 0, st>>>(part, p.nsplit, p.ld, p.nout, nullptr, c.scale, c.dtype, c.out, c.out_lse);
}
