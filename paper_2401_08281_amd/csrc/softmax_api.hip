// Host runtime and C ABI of libvs_softmax (see include/vs_softmax.h for the contract).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/vs_softmax.h"
#include "softmax.hpp"

namespace {

thread_local char g_err[512] = "";

int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? VS_OK : fail(VS_ERR_DEVICE, "%s: %s", who, hipGetErrorString(e));
}

struct Carver {
  int64_t off = 0;
  int64_t take(int64_t bytes) { const int64_t o = off; off = (off + bytes + 255) / 256 * 256; return o; }
};
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
inline int64_t elem_bytes(int dtype) { return dtype == VS_FP32 ? 4 : 2; }
inline SmForm form_of(int dtype) { return SmForm{dtype, dtype == VS_FP32 ? 2 : 1}; }

// Work space that records and kept scores of a piece of the queries may take, and the two copies of a piece of G: what
// the 256 MB last-level cache still holds when the products read it.
constexpr int64_t kPieceBytes = 256 << 20;

// fp16 and bf16 rows of whole K blocks are multiplied as they are; others through prepared copies
bool rows_direct(int dtype, int d) { return dtype != VS_FP32 && d % 64 == 0; }

struct LogprobPlan {
  SmForm f;
  bool few, direct, keep;
  int64_t parts, keep_ld, piece;
  int64_t kblocks, row_bytes;
  int64_t o_x, o_xs, o_q, o_qs, o_rec, o_keep, bytes;
};

LogprobPlan logprob_plan(int64_t nb, int64_t nq, int d, int dtype, int k) {
  LogprobPlan p{};
  p.f = form_of(dtype);
  p.direct = rows_direct(dtype, d);
  // Few queries: rows streamed past all of them, or tiles.  Streamed rows need no prepared copies and no LDS, and fp32
  // ones are multiplied once instead of three times; tiles read a row's fragment once for 128 queries.  Streamed and tiles
  // in us, k = 5: fp32 100,000 x 768, 16 queries 74 and 251, 64 queries 194 and 306; bf16 100,000 x 100 (copies) 64
  // queries 34 and 60; bf16 100,000 x 768 (none) 16 queries 41 and 44, 32 queries 47 and 44, 64 queries 81 and 66;
  // 100,000 x 320 32 queries 28 and 32, 64 queries 48 and 45.
  p.few = nq <= (p.direct ? kSmFewQueries / 2 : kSmFewQueries);
  p.parts = (nb + kSmRecRows - 1) / kSmRecRows;
  p.keep_ld = round_up(nb, kSmTileRows);
  // A record that holds two of the k best costs its 128 scores again, and k^2 / (2 parts) records do on average; kept scores
  // cost 8 bytes of traffic each and a selection over all of them.  Recomputed and kept in us: 1000 queries, d = 128, bf16:
  // 2500 rows, k = 10 (2 records for each of the k) 58 and 39, 4000 rows (3.1) 52 and 44, 10,000 rows, k = 20 (3.9) 65 and
  // 63, k = 10 (7.8) 50 and 59, 65,536 rows, k = 64 (8) 182 and 952; 64 queries, 8000 rows, k = 32 (2) 88 and 38.
  p.keep = k > 0 && p.parts <= 3 * (int64_t)k;
  const int64_t per = p.parts * (int64_t)sizeof(float4) + (p.keep ? p.keep_ld * 4 : 0);
  p.piece = std::min(nq, std::max<int64_t>(kSmTileQueries, per > 0 ? kPieceBytes / per / kSmTileQueries * kSmTileQueries : nq));
  p.kblocks = p.f.blocks(d);
  p.row_bytes = p.direct ? d * elem_bytes(dtype) : p.kblocks * 128;
  Carver c;
  if (!p.few && !p.direct) {
    p.o_x = c.take(nb * p.row_bytes);
    p.o_xs = c.take(nb * 4);
    p.o_q = c.take(nq * p.row_bytes);
    p.o_qs = c.take(nq * 4);
  }
  p.o_rec = c.take(p.piece * p.parts * (int64_t)sizeof(float4));
  p.o_keep = c.take(p.keep ? p.piece * p.keep_ld * 4 : 0);
  p.bytes = c.off;
  return p;
}

struct GradPlan {
  SmForm f;
  bool direct, small;
  int64_t tile_q, kblocks, row_bytes, chunk, ld, g_row, gt_row, xt_row, qt_row;
  SmProductPlan to_q, to_x;
  int64_t o_x, o_xs, o_q, o_qs, o_xt, o_xts, o_qt, o_qts, o_cm, o_coef, o_bound, o_g, o_gt, o_dq, o_dx, o_db, bytes;
};

GradPlan grad_plan(int64_t nb, int64_t nq, int d, int dtype) {
  GradPlan p{};
  p.f = form_of(dtype);
  p.direct = rows_direct(dtype, d);
  p.kblocks = p.f.blocks(d);
  p.row_bytes = p.direct ? d * elem_bytes(dtype) : p.kblocks * 128;
  const int64_t el = 2 * p.f.planes;
  const int64_t nqp = round_up(nq, kSmTileQueries), nbp = round_up(nb, kSmTileRows);
  p.chunk = std::min(nbp, std::max<int64_t>(kSmTileRows, kPieceBytes / (2 * el * nqp) / kSmTileRows * kSmTileRows));
  p.small = sm_gradients_small(p.f, p.chunk, nq, p.kblocks);
  p.tile_q = p.small ? 64 : kSmTileQueries;
  p.ld = round_up(d, 4);
  p.g_row = p.chunk * el;
  p.gt_row = nqp * el;
  p.xt_row = p.f.blocks(nb) * 128;
  p.qt_row = p.f.blocks(nq) * 128;
  p.to_q = plan_sm_product(d, nq, p.f.blocks(p.chunk));
  p.to_x = plan_sm_product(d, p.chunk, p.f.blocks(nq));
  Carver c;
  if (!p.direct) {
    p.o_x = c.take(nb * p.row_bytes);
    p.o_xs = c.take(nb * 4);
    p.o_q = c.take(nq * p.row_bytes);
    p.o_qs = c.take(nq * 4);
  }
  p.o_xt = c.take(d * p.xt_row);
  p.o_xts = c.take((int64_t)d * 4);
  p.o_qt = c.take(d * p.qt_row);
  p.o_qts = c.take((int64_t)d * 4);
  p.o_cm = c.take((int64_t)d * 8);
  p.o_coef = c.take(nq * (int64_t)sizeof(float4));
  p.o_bound = c.take(nq * 4);
  p.o_g = c.take(nq * p.g_row);
  p.o_gt = c.take(p.chunk * p.gt_row);
  p.o_dq = c.take(p.to_q.splits * nq * p.ld * 4);
  p.o_dx = c.take(!p.to_x.big || p.to_x.splits > 1 ? p.to_x.splits * p.chunk * p.ld * 4 : 0);
  p.o_db = c.take(nqp / p.tile_q * p.chunk * 4);
  p.bytes = c.off;
  return p;
}

int check_rows(const char* who, int64_t nb, int64_t nq, int d, int dtype) {
  if (d < 1 || d > VS_MAX_ROW) return fail(VS_ERR_INVALID_ARG, "%s: d = %d outside [1, %d]", who, d, VS_MAX_ROW);
  if (nb < 0 || nb >= (int64_t)1 << 31) return fail(VS_ERR_INVALID_ARG, "%s: nb = %lld outside [0, 2^31)", who, (long long)nb);
  if (nq < 0 || nq >= (int64_t)1 << 31) return fail(VS_ERR_INVALID_ARG, "%s: nq = %lld outside [0, 2^31)", who, (long long)nq);
  if (dtype < VS_FP32 || dtype > VS_BF16) return fail(VS_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  return VS_OK;
}

int check_space(const char* who, const void* ws, int64_t have, int64_t need) {
  if (need > 0 && !ws) return fail(VS_ERR_INVALID_ARG, "%s: no work space (%lld bytes)", who, (long long)need);
  if (have < need) return fail(VS_ERR_INVALID_ARG, "%s: work space of %lld bytes, %lld needed", who, (long long)have, (long long)need);
  if (need > 0 && misaligned(ws, 256)) return fail(VS_ERR_INVALID_ARG, "%s: work space is not 256-byte aligned", who);
  return VS_OK;
}

// ---- attention over the codes of an index ----------------------------------------
// (vs_ivfpq, defined in libvs, derives from the part of it that is read here, its first member)
const IvfStore* store_of(const vs_ivfpq* ix) { return reinterpret_cast<const IvfStore*>(ix); }

struct AttendSpace {
  AttendPlan plan;
  int nprobe = 0;                  // 0: all lists
  int64_t o_q32 = 0, o_probes = 0, o_part = 0, bytes = 0;
};

int attend_space(const char* who, const vs_ivfpq* ix, int64_t nq, int dk, int v0, int dtype, int nprobe, bool grad, AttendSpace* o) {
  if (!ix) return fail(VS_ERR_INVALID_ARG, "%s: index is null", who);
  const IvfStore& s = *store_of(ix);
  if (nq < 0 || nq >= (int64_t)1 << 31) return fail(VS_ERR_INVALID_ARG, "%s: nq = %lld outside [0, 2^31)", who, (long long)nq);
  if (dtype < VS_FP32 || dtype > VS_BF16) return fail(VS_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (s.g.metric != VS_METRIC_IP) return fail(VS_ERR_UNSUPPORTED, "%s: the index is not an inner-product index", who);
  if (s.g.nbits != 4) return fail(VS_ERR_UNSUPPORTED, "%s: the index has %d-bit codes (only 4)", who, s.g.nbits);
  if (dk < 1 || dk > s.g.d || dk % s.g.dsub) return fail(VS_ERR_INVALID_ARG, "%s: dk = %d is not a multiple of %d in [1, %d]", who, dk, s.g.dsub, s.g.d);
  if (v0 < 0 || v0 >= s.g.d || v0 % s.g.dsub) return fail(VS_ERR_INVALID_ARG, "%s: v0 = %d is not a multiple of %d in [0, %d)", who, v0, s.g.dsub, s.g.d);
  if (nprobe < 0 || nprobe > VS_MAX_K) return fail(VS_ERR_INVALID_ARG, "%s: nprobe = %d outside [0, %d]", who, nprobe, VS_MAX_K);
  o->nprobe = nprobe < s.g.nlist ? nprobe : 0;
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess || device != s.device) return fail(VS_ERR_INVALID_ARG, "%s: the index is on device %d, the current device is %d", who, s.device, device);
  o->plan = attend_plan(s.g, s.ntotal, nq, dk, v0, dtype, o->nprobe, grad);
  if (!o->plan.fits) return fail(VS_ERR_UNSUPPORTED, "%s: the tables of M = %d, d = %d exceed the on-chip memory", who, s.g.M, s.g.d);
  if ((nq + o->plan.qb - 1) / o->plan.qb * o->plan.nsplit >= (int64_t)1 << 31) return fail(VS_ERR_UNSUPPORTED, "%s: more than 2^31 workgroups", who);
  Carver c;
  if (o->nprobe > 0) {
    o->o_q32 = c.take(nq * s.g.d * 4);
    o->o_probes = c.take(nq * o->nprobe * 4);
  }
  o->o_part = c.take(nq * o->plan.nsplit * o->plan.ld * 4);
  o->bytes = c.off;
  return VS_OK;
}

int attend_run(const char* who, const vs_ivfpq* ix, AttendCall& c, const AttendSpace& sp, bool grad, void* workspace,
               int64_t workspace_bytes, void* hip_stream) {
  if (misaligned(c.q, 16) || misaligned(c.g_out, 16)) return fail(VS_ERR_INVALID_ARG, "%s: vectors have to be 16-byte aligned", who);
  if (int rc = check_space(who, workspace, workspace_bytes, sp.bytes)) return rc;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(workspace);
  if (sp.nprobe > 0) {
    // (a replay could meet the index's work space at another size, or in use by another call)
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cs) != hipSuccess || cs != hipStreamCaptureStatusNone)
      return fail(VS_ERR_UNSUPPORTED, "%s: probed lists under capture (the coarse quantizer uses the index's own work space)", who);
    float* q32 = reinterpret_cast<float*>(ws + sp.o_q32);
    int32_t* probes = reinterpret_cast<int32_t*>(ws + sp.o_probes);
    launch_attend_pad(c.q, c.nq, c.dk, c.ix->g.d, c.dtype, q32, st);
    if (int rc = vs_ivfpq_coarse(ix, q32, c.nq, sp.nprobe, probes, nullptr, hip_stream)) return fail(rc, "%s: %s", who, vs_last_error());
    c.probes = probes;
    c.nprobe = sp.nprobe;
  }
  launch_attend(c, sp.plan, grad, reinterpret_cast<float*>(ws + sp.o_part), st);
  return launched(who);
}

}  // namespace

extern "C" {

const char* vs_softmax_last_error(void) { return g_err; }

int64_t vs_flat_logprob_workspace_bytes(int64_t nb, int64_t nq, int32_t d, int32_t dtype, int32_t k) {
  const char* who = "vs_flat_logprob_workspace_bytes";
  if (check_rows(who, nb, nq, d, dtype)) return -1;
  if (k < 0 || k > VS_MAX_TOP) { fail(VS_ERR_INVALID_ARG, "%s: k = %d outside [0, %d]", who, k, VS_MAX_TOP); return -1; }
  return logprob_plan(nb, nq, d, dtype, k).bytes;
}

int vs_flat_logprob(const void* x, int64_t nb, const void* q, int64_t nq, int32_t d, int32_t dtype, float scale,
                    const float* bias, const int64_t* targets, int32_t nt, int32_t k, float* out_logp, float* out_lse,
                    float* out_entropy, float* out_top_logp, int64_t* out_top_ids, void* workspace,
                    int64_t workspace_bytes, void* hip_stream) {
  const char* who = "vs_flat_logprob";
  if (int rc = check_rows(who, nb, nq, d, dtype)) return rc;
  if (nt < 0) return fail(VS_ERR_INVALID_ARG, "%s: nt = %d", who, nt);
  if (k < 0 || k > VS_MAX_TOP) return fail(VS_ERR_INVALID_ARG, "%s: k = %d outside [0, %d]", who, k, VS_MAX_TOP);
  if (!std::isfinite(scale)) return fail(VS_ERR_INVALID_ARG, "%s: scale is not finite", who);
  if (nq == 0) return VS_OK;
  if (!q || (nb > 0 && !x) || !out_lse || !out_entropy || (nt > 0 && (!targets || !out_logp)) ||
      (k > 0 && (!out_top_logp || !out_top_ids)))
    return fail(VS_ERR_INVALID_ARG, "%s: null pointer", who);
  if (misaligned(x, 16) || misaligned(q, 16)) return fail(VS_ERR_INVALID_ARG, "%s: x and q have to be 16-byte aligned", who);
  const LogprobPlan p = logprob_plan(nb, nq, d, dtype, k);
  if (int rc = check_space(who, workspace, workspace_bytes, p.bytes)) return rc;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(workspace);
  SmScores s;
  s.kunits = 2 * p.kblocks; s.nx = nb; s.bias = bias; s.scale = scale;
  s.x = SmMatrix{x, p.row_bytes, nb, nullptr};
  s.q = SmMatrix{q, p.row_bytes, nq, nullptr};
  if (!p.few && !p.direct && nb > 0) {
    SmSide sx, sq;
    sx.x = x; sx.n = nb; sx.bias = bias; sx.rows = ws + p.o_x; sx.row_scale = reinterpret_cast<float*>(ws + p.o_xs);
    sq.x = q; sq.n = nq; sq.rows = ws + p.o_q; sq.row_scale = reinterpret_cast<float*>(ws + p.o_qs);
    launch_sm_prep_rows(p.f, sx, sq, d, st);
    s.x = SmMatrix{sx.rows, p.row_bytes, nb, sx.row_scale};
    s.q = SmMatrix{sq.rows, p.row_bytes, nq, sq.row_scale};
    s.raw_x = x; s.d = d; s.dtype = dtype;
  }
  SmRecords r;
  r.rec = reinterpret_cast<float4*>(ws + p.o_rec);
  r.parts = p.parts;
  r.keep = p.keep && nb > 0 ? reinterpret_cast<float*>(ws + p.o_keep) : nullptr;
  r.keep_ld = p.keep_ld;
  const SmMatrix qs = s.q;
  for (int64_t q0 = 0; q0 < nq; q0 += p.piece) {
    const int64_t n = std::min(p.piece, nq - q0);
    const char* qp = static_cast<const char*>(q) + q0 * d * elem_bytes(dtype);
    if (nb > 0) {
      if (p.few) {
        launch_sm_scores_few(dtype, x, nb, qp, n, d, scale, bias, r, k > 0 && !p.keep, st);
      } else {
        s.q = SmMatrix{static_cast<const char*>(qs.p) + q0 * qs.row_bytes, qs.row_bytes, n, qs.scale ? qs.scale + q0 : nullptr};
        s.nq = n;
        s.raw_q = qp;
        launch_sm_scores(p.f, p.direct, s, r, k > 0 && !p.keep, st);
      }
    }
    SmFinish fin{x, nb, qp, n, d, dtype, scale, bias, targets ? targets + q0 * nt : nullptr, nt, k,
                 out_logp ? out_logp + q0 * nt : nullptr, out_lse + q0, out_entropy + q0,
                 out_top_logp ? out_top_logp + q0 * k : nullptr, out_top_ids ? out_top_ids + q0 * k : nullptr};
    launch_sm_finish(fin, r, st);
  }
  return launched(who);
}

int64_t vs_flat_logprob_grad_workspace_bytes(int64_t nb, int64_t nq, int32_t d, int32_t dtype) {
  if (check_rows("vs_flat_logprob_grad_workspace_bytes", nb, nq, d, dtype)) return -1;
  if (nb == 0 || nq == 0) return 0;
  return grad_plan(nb, nq, d, dtype).bytes;
}

int vs_flat_logprob_grad(const void* x, int64_t nb, const void* q, int64_t nq, int32_t d, int32_t dtype, float scale,
                         const float* bias, const int64_t* targets, int32_t nt, const float* lse, const float* entropy,
                         const float* g_logp, const float* g_lse, const float* g_entropy, void* out_dq, void* out_dx,
                         float* out_dbias, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  const char* who = "vs_flat_logprob_grad";
  if (int rc = check_rows(who, nb, nq, d, dtype)) return rc;
  if (nt < 0) return fail(VS_ERR_INVALID_ARG, "%s: nt = %d", who, nt);
  if (!std::isfinite(scale)) return fail(VS_ERR_INVALID_ARG, "%s: scale is not finite", who);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (nb == 0 || nq == 0) {
    if (out_dq) launch_sm_zero(out_dq, nq * d * elem_bytes(dtype), st);
    if (out_dx) launch_sm_zero(out_dx, nb * d * elem_bytes(dtype), st);
    if (out_dbias) launch_sm_zero(out_dbias, nb * 4, st);
    return launched(who);
  }
  if (!x || !q || !lse || (g_logp && nt > 0 && !targets)) return fail(VS_ERR_INVALID_ARG, "%s: null pointer", who);
  if (g_entropy && !entropy) return fail(VS_ERR_INVALID_ARG, "%s: g_entropy without entropy", who);
  if (misaligned(x, 16) || misaligned(q, 16) || misaligned(out_dq, 4) || misaligned(out_dx, 4))
    return fail(VS_ERR_INVALID_ARG, "%s: x and q have to be 16-byte aligned, their gradients 4-byte", who);
  const GradPlan p = grad_plan(nb, nq, d, dtype);
  if (int rc = check_space(who, workspace, workspace_bytes, p.bytes)) return rc;
  // (far beyond what the work space of such a call leaves of the memory)
  const int64_t tiles = round_up(nq, p.tile_q) / p.tile_q * (p.chunk / (p.small ? 128 : kSmTileRows));
  if (std::max(tiles, std::max(p.to_q.groups, p.to_x.groups)) >= kGroupsInRow)
    return fail(VS_ERR_UNSUPPORTED, "%s: more than 2^23 tiles", who);
  if (!out_dq && !out_dx && !out_dbias) return VS_OK;
  char* ws = static_cast<char*>(workspace);
  auto at = [&](int64_t o) { return reinterpret_cast<float*>(ws + o); };
  const SmForm prod{VS_FP16, p.f.planes};                    // the operands of the two products are fp16 parts
  float* bound = at(p.o_bound);
  SmGrads g{lse, entropy, targets, nt, nt > 0 ? g_logp : nullptr, g_lse, g_entropy};
  u32* colmax = reinterpret_cast<u32*>(ws + p.o_cm);
  launch_sm_coefs(g, nq, nb, reinterpret_cast<float4*>(ws + p.o_coef), bound, colmax, 2 * d, st);
  SmSide sx, sq;
  sx.x = x; sx.n = nb; sx.bias = bias; sx.rows = ws + p.o_x; sx.row_scale = at(p.o_xs);
  sx.cols = ws + p.o_xt; sx.col_scale = at(p.o_xts); sx.colmax = colmax;
  sq.x = q; sq.n = nq; sq.factor = bound; sq.rows = ws + p.o_q; sq.row_scale = at(p.o_qs);
  sq.cols = ws + p.o_qt; sq.col_scale = at(p.o_qts); sq.colmax = colmax + d;
  SmScores s;
  s.kunits = 2 * p.kblocks; s.nq = nq; s.scale = scale;
  const char* xp = static_cast<const char*>(x);
  const float* xs = nullptr;
  s.q = SmMatrix{q, p.row_bytes, nq, nullptr};
  if (!p.direct) {
    launch_sm_prep_rows(p.f, sx, sq, d, st);
    xp = ws + p.o_x; xs = at(p.o_xs);
    s.q = SmMatrix{sq.rows, p.row_bytes, nq, sq.row_scale};
    s.raw_q = q; s.d = d; s.dtype = dtype;
  }
  SmSide cx = sx, cq = sq;
  if (!out_dq) cx.n = 0;
  if (!out_dx) cq.n = 0;
  launch_sm_prep_cols(p.f, cx, cq, d, st);
  const float alpha = scale * (1.f / 16384.f);
  for (int64_t x0 = 0; x0 < nb; x0 += p.chunk) {
    const int64_t n = std::min(p.chunk, nb - x0);
    s.x = SmMatrix{xp + x0 * p.row_bytes, p.row_bytes, n, xs ? xs + x0 : nullptr};
    s.nx = n;
    if (!p.direct) s.raw_x = static_cast<const char*>(x) + x0 * d * elem_bytes(dtype);
    s.bias = bias ? bias + x0 : nullptr;
    SmGOut o{reinterpret_cast<float4*>(ws + p.o_coef), bound, targets, nt, g.g_logp, x0,
             out_dq ? ws + p.o_g : nullptr, p.g_row, out_dx ? ws + p.o_gt : nullptr, p.gt_row,
             out_dbias ? at(p.o_db) : nullptr, p.chunk, p.small};
    launch_sm_gradients(p.f, p.direct, s, o, st);
    if (out_dq) {
      const SmMatrix a{ws + p.o_xt + x0 / p.f.per_block() * 128, p.xt_row, d, nullptr}, b{ws + p.o_g, p.g_row, nq, nullptr};
      launch_sm_product(prod, p.to_q, a, b, p.f.blocks(n), x0 > 0, at(p.o_dq), p.ld, st);
    }
    if (out_dx) {
      const SmMatrix a{ws + p.o_qt, p.qt_row, d, nullptr}, b{ws + p.o_gt, p.gt_row, n, nullptr};
      char* dx = static_cast<char*>(out_dx) + x0 * d * elem_bytes(dtype);
      if (p.to_x.big && p.to_x.splits == 1) {
        launch_sm_product_direct(prod, a, b, p.f.blocks(nq), at(p.o_qts), alpha, s.bias, dtype, dx, st);
      } else {
        launch_sm_product(prod, p.to_x, a, b, p.f.blocks(nq), false, at(p.o_dx), p.ld, st);
        launch_sm_product_out(at(p.o_dx), p.to_x.splits, n, p.ld, d, at(p.o_qts), nullptr, alpha, s.bias, dtype, dx, st);
      }
    }
    if (out_dbias) launch_sm_sum_parts(at(p.o_db), (nq + p.tile_q - 1) / p.tile_q, p.chunk, n, out_dbias + x0, st);
  }
  if (out_dq) launch_sm_product_out(at(p.o_dq), p.to_q.splits, nq, p.ld, d, at(p.o_xts), bound, alpha, nullptr, dtype, out_dq, st);
  return launched(who);
}

int64_t vs_ivfpq_attend_workspace_bytes(const vs_ivfpq* ix, int64_t nq, int32_t dk, int32_t v0, int32_t dtype, int32_t nprobe) {
  AttendSpace sp;
  return attend_space("vs_ivfpq_attend_workspace_bytes", ix, nq, dk, v0, dtype, nprobe, false, &sp) ? -1 : sp.bytes;
}

int vs_ivfpq_attend(const vs_ivfpq* ix, const void* q, int64_t nq, int32_t dk, int32_t v0, int32_t dtype, int32_t nprobe,
                    float scale, const int64_t* limits, void* out, float* out_lse, void* workspace, int64_t workspace_bytes,
                    void* hip_stream) {
  const char* who = "vs_ivfpq_attend";
  AttendSpace sp;
  if (int rc = attend_space(who, ix, nq, dk, v0, dtype, nprobe, false, &sp)) return rc;
  if (!std::isfinite(scale)) return fail(VS_ERR_INVALID_ARG, "%s: scale is not finite", who);
  if (nq == 0) return VS_OK;
  if (!q || !out) return fail(VS_ERR_INVALID_ARG, "%s: null pointer", who);
  AttendCall c{store_of(ix), q, nq, dk, v0, dtype, scale, limits, nullptr, 0, nullptr, nullptr, nullptr, out, out_lse};
  return attend_run(who, ix, c, sp, false, workspace, workspace_bytes, hip_stream);
}

int64_t vs_ivfpq_attend_grad_workspace_bytes(const vs_ivfpq* ix, int64_t nq, int32_t dk, int32_t v0, int32_t dtype, int32_t nprobe) {
  AttendSpace sp;
  return attend_space("vs_ivfpq_attend_grad_workspace_bytes", ix, nq, dk, v0, dtype, nprobe, true, &sp) ? -1 : sp.bytes;
}

int vs_ivfpq_attend_grad(const vs_ivfpq* ix, const void* q, int64_t nq, int32_t dk, int32_t v0, int32_t dtype, int32_t nprobe,
                         float scale, const int64_t* limits, const float* lse, const void* g_out, const float* g_lse,
                         void* out_dq, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  const char* who = "vs_ivfpq_attend_grad";
  AttendSpace sp;
  if (int rc = attend_space(who, ix, nq, dk, v0, dtype, nprobe, true, &sp)) return rc;
  if (!std::isfinite(scale)) return fail(VS_ERR_INVALID_ARG, "%s: scale is not finite", who);
  if (nq == 0) return VS_OK;
  if (!q || !lse || !g_out || !out_dq) return fail(VS_ERR_INVALID_ARG, "%s: null pointer", who);
  AttendCall c{store_of(ix), q, nq, dk, v0, dtype, scale, limits, nullptr, 0, lse, g_out, g_lse, out_dq, nullptr};
  return attend_run(who, ix, c, sp, true, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
