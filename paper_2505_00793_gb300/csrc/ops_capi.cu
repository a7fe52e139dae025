// C entry points of the operators on packed token rows (mixflow.h): argument checks, the
// rotary rates, launches.
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/mixflow.h"
#include "attn_ops.h"

namespace {

using mf::AttnParams;
using mf::EmbedParams;
using mf::RopeParams;

bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A row buffer: on a 16-byte boundary, its leading dimension a multiple of 8 elements that
// holds cols, and its byte offsets within 63 bits.
bool rows_ok(const void* p, int64_t ld, int64_t cols, int64_t rows) {
  return p && aligned(p) && ld >= cols && ld % 8 == 0 && ld <= (int64_t{1} << 38) &&
         ld <= (int64_t{1} << 60) / (rows > 0 ? rows : 1);
}
bool both(const void* a, const void* b) { return (a == nullptr) == (b == nullptr); }

// Sequences of n_rows rows; with every_row a batch without sequences is one of them.
bool make_seq(int64_t n_rows, const int32_t* start, int n_seq, bool every_row, mf::SeqRows* s) {
  if (n_rows < 0 || n_rows > INT32_MAX - 256 || n_seq < 0 || n_seq == INT32_MAX) return false;
  if (every_row && !start && n_seq == 0) n_seq = 1;
  if (n_seq < 1 || (!start && n_rows % n_seq)) return false;
  s->start = start;
  s->n = n_seq;
  s->rows = static_cast<int>(n_rows);
  s->len = start ? 0 : static_cast<int>(n_rows / n_seq);
  return true;
}

bool heads_ok(int Hq, int Hkv, int Hc, int D) {
  return Hq >= 1 && Hkv >= 1 && Hc >= 0 && D >= 8 && D <= 128 && D % 8 == 0 && Hq <= 65536 &&
         Hkv <= 65536 && Hc <= 65536;
}

bool finite(float x) { return isfinite(x); }

// Rates of the rotated pairs, in units of 2^-64 turns a position.
bool make_rope(const mf_rope_desc& r, int D, RopeParams* p) {
  const int R = r.dims == 0 ? D : r.dims;
  if (r.layout != MF_ROPE_HALF && r.layout != MF_ROPE_INTERLEAVED) return false;
  if (R < 2 || R > D || R % 2) return false;
  if (!finite(r.base) || r.base < 0.f || !finite(r.mscale)) return false;
  double base = r.base > 0.f ? r.base : 10000.0;
  const double f = r.factor;
  switch (r.scaling) {
    case MF_ROPE_SCALE_NONE:
      break;
    case MF_ROPE_SCALE_BASE:
      if (R <= 2) return false;
      [[fallthrough]];
    case MF_ROPE_SCALE_LINEAR:
      if (!finite(r.factor) || f <= 0.0) return false;
      break;
    case MF_ROPE_SCALE_BANDS:
      if (!finite(r.factor) || f <= 0.0 || r.orig_len < 1 || !(r.low_turns >= 0.f) ||
          !(r.high_turns > r.low_turns) || !finite(r.high_turns))
        return false;
      break;
    default:
      return false;
  }
  if (r.scaling == MF_ROPE_SCALE_BASE) base *= pow(f, static_cast<double>(R) / (R - 2));
  constexpr double kTurn = 6.283185307179586476925;
  for (int j = 0; j < R / 2; ++j) {
    double w = pow(base, -2.0 * j / R);
    if (r.scaling == MF_ROPE_SCALE_LINEAR) w /= f;
    if (r.scaling == MF_ROPE_SCALE_BANDS) {
      const double turns = r.orig_len * w / kTurn;
      double keep = (turns - r.low_turns) / (static_cast<double>(r.high_turns) - r.low_turns);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      w = keep * w + (1.0 - keep) * w / f;
    }
    // whole turns a position do not move the angle
    double turns = w / kTurn;
    if (!isfinite(turns)) return false;
    turns -= floor(turns);
    p->phase[j] = static_cast<uint64_t>(ldexp(turns, 64) < 18446744073709551615.0 ? ldexp(turns, 64) : 0.0);
  }
  p->R = R;
  p->half = r.layout == MF_ROPE_HALF;
  p->mscale = r.mscale == 0.f ? 1.f : r.mscale;
  return true;
}

mf_status done(cudaError_t e) {
  if (e == cudaSuccess) return MF_OK;
  if (e == cudaErrorInvalidValue) {
    cudaGetLastError();
    return MF_ERR_INVALID_ARG;
  }
  return MF_ERR_CUDA;
}

// Partial sums of two gains' gradients, and with tangents of theirs.
size_t rope_work(const mf_qk_rope_args& a, bool dual) {
  return static_cast<size_t>(mf::kRopeMaxBlocks) * (dual ? 4 : 2) * a.head_dim * sizeof(float);
}

// Checks what the two passes share and fills the kernels' parameters.
mf_status rope_params(const mf_qk_rope_args& a, RopeParams* p) {
  const bool bf = MF_PREC_BF16 == a.y_prec, xbf = MF_PREC_BF16 == a.x_prec;
  if ((!bf && a.y_prec != MF_PREC_FP32) || (!xbf && a.x_prec != MF_PREC_FP32)) return MF_ERR_INVALID_ARG;
  if (!heads_ok(a.n_heads, a.n_kv_heads, a.n_copy_heads, a.head_dim)) return MF_ERR_INVALID_ARG;
  if (!make_seq(a.n_rows, a.seq_start, a.n_seq, a.pos != nullptr, &p->seq)) return MF_ERR_INVALID_ARG;
  if (!make_rope(a.rope, a.head_dim, p)) return MF_ERR_INVALID_ARG;
  if (!both(a.gq, a.gk) || !both(a.gqd, a.gkd) || (a.gqd && !a.gq)) return MF_ERR_INVALID_ARG;
  if (a.gq && (!finite(a.eps) || a.eps < 0.f)) return MF_ERR_INVALID_ARG;
  for (const float* g : {a.gq, a.gk, a.gqd, a.gkd})
    if (!aligned(g)) return MF_ERR_INVALID_ARG;
  if (xbf && !bf) return MF_ERR_UNSUPPORTED;
  p->Hq = a.n_heads;
  p->Hkv = a.n_kv_heads;
  p->Hc = a.n_copy_heads;
  p->D = a.head_dim;
  p->eps = a.eps;
  p->x = a.x; p->xd = a.xd; p->ldx = a.ldx;
  p->gq = a.gq; p->gk = a.gk; p->gqd = a.gqd; p->gkd = a.gkd;
  p->pos = a.pos;
  p->status = a.status;
  return MF_OK;
}

// A buffer that is written may be the one that it comes from, and nothing else.
bool in_place_ok(const void* in, int64_t ldin, const void* out, int64_t ldout, bool same_type) {
  return in != out || (ldin == ldout && same_type);
}

// Whether no output begins where another buffer of the call does.  (More cannot be told from
// addresses: column ranges of one buffer of rows interleave.)
bool outputs_apart(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* const* o = outs.begin(); o != outs.end(); ++o) {
    if (!*o) continue;
    for (const void* const* q = outs.begin(); q != o; ++q)
      if (*q == *o) return false;
    for (const void* i : ins)
      if (i == *o) return false;
  }
  return true;
}

size_t attn_work(const mf_attn_args& a) {
  return static_cast<size_t>(a.n_rows) * a.n_heads * sizeof(float) * (a.qd ? 2 : 1);
}
// Behind that, on a 16-byte boundary, the sums of sinks.
size_t window_work(const mf_attn_args& a, int64_t window, int sinks) {
  const size_t rows = (attn_work(a) + 15) / 16 * 16;
  const bool all = window >= a.n_rows;           // plain attention
  return rows + (all ? 0 : sizeof(float) * mf::window_part(a.n_rows, a.n_kv_heads, a.head_dim,
                                                           static_cast<int>(window), sinks, a.qd != nullptr));
}

mf_status attn_params(const mf_attn_args& a, bool bwd, AttnParams* p, size_t work) {
  if (!heads_ok(a.n_heads, a.n_kv_heads, 0, a.head_dim) || a.n_heads % a.n_kv_heads)
    return MF_ERR_INVALID_ARG;
  if (!make_seq(a.n_rows, a.seq_start, a.n_seq, false, &p->seq)) return MF_ERR_INVALID_ARG;
  if (!finite(a.scale) || a.scale < 0.f) return MF_ERR_INVALID_ARG;
  const bool dual = a.qd != nullptr;
  for (const void* t : {a.kd, a.vd, static_cast<const void*>(a.od), static_cast<const void*>(a.rbar)})
    if ((t != nullptr) != dual) return MF_ERR_INVALID_ARG;
  if (bwd)
    for (const void* t : {a.d_od, static_cast<const void*>(a.dqd), static_cast<const void*>(a.dkd),
                          static_cast<const void*>(a.dvd)})
      if ((t != nullptr) != dual) return MF_ERR_INVALID_ARG;
  if (a.n_rows == 0) return MF_OK;
  const int64_t N = a.n_rows, cq = static_cast<int64_t>(a.n_heads) * a.head_dim;
  const int64_t ck = static_cast<int64_t>(a.n_kv_heads) * a.head_dim;
  bool ok = rows_ok(a.q, a.ldq, cq, N) && rows_ok(a.k, a.ldk, ck, N) && rows_ok(a.v, a.ldv, ck, N) &&
            rows_ok(a.o, a.ldo, cq, N) && a.lse;
  if (dual)
    ok = ok && aligned(a.qd) && aligned(a.kd) && aligned(a.vd) && aligned(a.od);
  if (bwd) {
    ok = ok && rows_ok(a.d_o, a.lddo, cq, N) && rows_ok(a.dq, a.lddq, cq, N) &&
         rows_ok(a.dk, a.lddk, ck, N) && rows_ok(a.dv, a.lddv, ck, N) && a.work && aligned(a.work);
    if (dual) ok = ok && aligned(a.d_od) && aligned(a.dqd) && aligned(a.dkd) && aligned(a.dvd);
    ok = ok && a.work_bytes >= work;
  }
  if (!ok) return MF_ERR_INVALID_ARG;
  if (dual && a.head_dim > 64) return MF_ERR_UNSUPPORTED;
  if (bwd ? !outputs_apart({a.dq, a.dk, a.dv, a.dqd, a.dkd, a.dvd, a.work},
                           {a.q, a.k, a.v, a.qd, a.kd, a.vd, a.o, a.od, a.d_o, a.d_od, a.lse, a.rbar})
          : !outputs_apart({a.o, a.od, a.lse, a.rbar}, {a.q, a.k, a.v, a.qd, a.kd, a.vd}))
    return MF_ERR_INVALID_ARG;
  auto cb = [](const void* x) { return static_cast<const __nv_bfloat16*>(x); };
  auto mb = [](void* x) { return static_cast<__nv_bfloat16*>(x); };
  p->Hq = a.n_heads; p->Hkv = a.n_kv_heads; p->D = a.head_dim;
  p->scale = a.scale > 0.f ? a.scale : 1.f / sqrtf(static_cast<float>(a.head_dim));
  p->q = cb(a.q); p->k = cb(a.k); p->v = cb(a.v);
  p->qd = cb(a.qd); p->kd = cb(a.kd); p->vd = cb(a.vd);
  p->o = mb(a.o); p->od = mb(a.od);
  p->ldq = a.ldq; p->ldk = a.ldk; p->ldv = a.ldv; p->ldo = a.ldo;
  p->lse = a.lse; p->rbar = a.rbar;
  p->status = a.status;
  if (bwd) {
    p->d_o = cb(a.d_o); p->d_od = cb(a.d_od); p->lddo = a.lddo;
    p->dq = mb(a.dq); p->dk = mb(a.dk); p->dv = mb(a.dv);
    p->dqd = mb(a.dqd); p->dkd = mb(a.dkd); p->dvd = mb(a.dvd);
    p->lddq = a.lddq; p->lddk = a.lddk; p->lddv = a.lddv;
    p->Dr = static_cast<float*>(a.work);
    p->Drd = dual ? p->Dr + static_cast<int64_t>(a.n_heads) * N : nullptr;
  }
  return MF_OK;
}

mf_status attn_window(const mf_attn_args* args, int64_t window, int n_sink, bool bwd, void* stream) {
  if (!args || window < 1 || n_sink < 0) return MF_ERR_INVALID_ARG;
  const mf_attn_args& a = *args;
  AttnParams p;
  const bool sized = n_sink <= mf::kMaxSinks && a.n_rows >= 0 && a.n_rows <= INT32_MAX - 256 &&
                     heads_ok(a.n_heads, a.n_kv_heads, 0, a.head_dim);    // else refused below
  const size_t work = sized ? window_work(a, window, n_sink) : 0;
  const mf_status st = attn_params(a, bwd, &p, work);
  if (st != MF_OK) return st;
  if (n_sink > mf::kMaxSinks) return MF_ERR_UNSUPPORTED;
  if (a.n_rows == 0) return MF_OK;
  const bool dual = a.qd != nullptr;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  // a window that holds every row is no window: the kernels without one
  if (window >= a.n_rows) return done(bwd ? mf::attn_tc_bwd(p, dual, s) : mf::attn_tc_fwd(p, dual, s));
  p.window = static_cast<int>(window);
  p.sinks = n_sink;
  if (bwd) p.part = reinterpret_cast<float*>(static_cast<char*>(a.work) + (attn_work(a) + 15) / 16 * 16);
  return done(bwd ? mf::attn_window_bwd(p, dual, s) : mf::attn_window_fwd(p, dual, s));
}

bool embed_sizes_ok(const mf_embed_args& a) {
  return a.n_rows >= 0 && a.n_rows <= INT32_MAX - 256 && a.vocab >= 1 && a.vocab <= INT32_MAX - 256 &&
         a.dim >= 1 && a.dim <= (1 << 20);
}
// Without rows dyd may be null where dEd is given.
size_t embed_work(const mf_embed_args& a) {
  return static_cast<size_t>(mf::embed_plan(a.n_rows, a.vocab, a.dim, a.dyd || a.dEd).bytes);
}
bool prec_ok(int p) { return p == MF_PREC_FP32 || p == MF_PREC_BF16; }

mf_status embed_params(const mf_embed_args& a, EmbedParams* p) {
  if (!embed_sizes_ok(a) || !prec_ok(a.y_prec) || !finite(a.scale)) return MF_ERR_INVALID_ARG;
  if (!make_seq(a.n_rows, a.seq_start, a.n_seq, true, &p->seq)) return MF_ERR_INVALID_ARG;
  if (a.n_rows > 0 && !a.ids) return MF_ERR_INVALID_ARG;
  p->vocab = static_cast<int>(a.vocab);
  p->dim = static_cast<int>(a.dim);
  p->scale = a.scale;
  p->ids = a.ids;
  return MF_OK;
}

}  // namespace

bool mf::rope_desc_ok(const mf_rope_desc& r, int D) {
  RopeParams p;
  return make_rope(r, D, &p);
}

extern "C" {

mf_status mf_qk_rope_work_bytes(const mf_qk_rope_args* args, size_t* bytes) {
  if (!args || !bytes || !heads_ok(args->n_heads, args->n_kv_heads, args->n_copy_heads, args->head_dim))
    return MF_ERR_INVALID_ARG;
  *bytes = rope_work(*args, args->dyd || args->xd);   // xd: asked with the forward's arguments
  return MF_OK;
}

mf_status mf_qk_rope_fwd(const mf_qk_rope_args* args, void* stream) {
  if (!args) return MF_ERR_INVALID_ARG;
  const mf_qk_rope_args& a = *args;
  RopeParams p;
  const mf_status st = rope_params(a, &p);
  if (st != MF_OK) return st;
  if (!both(a.xd, a.yd) || (a.gqd && !a.xd)) return MF_ERR_INVALID_ARG;
  if (a.n_rows == 0) return MF_OK;
  const int64_t cols = static_cast<int64_t>(a.n_heads + a.n_kv_heads + a.n_copy_heads) * a.head_dim;
  if (!rows_ok(a.x, a.ldx, cols, a.n_rows) || !rows_ok(a.y, a.ldy, cols, a.n_rows) || !aligned(a.xd) ||
      !aligned(a.yd) || !in_place_ok(a.x, a.ldx, a.y, a.ldy, a.x_prec == a.y_prec) ||
      (a.xd && !in_place_ok(a.xd, a.ldx, a.yd, a.ldy, a.x_prec == a.y_prec)))
    return MF_ERR_INVALID_ARG;
  if (!outputs_apart({a.y, a.yd}, {a.y == a.x ? nullptr : a.x, a.yd == a.xd ? nullptr : a.xd}))
    return MF_ERR_INVALID_ARG;
  p.y = a.y; p.yd = a.yd; p.ldy = a.ldy;
  return done(mf::qk_rope(p, false, a.x_prec == MF_PREC_BF16, a.y_prec == MF_PREC_BF16,
                          static_cast<cudaStream_t>(stream)));
}

mf_status mf_qk_rope_bwd(const mf_qk_rope_args* args, void* stream) {
  if (!args) return MF_ERR_INVALID_ARG;
  const mf_qk_rope_args& a = *args;
  RopeParams p;
  const mf_status st = rope_params(a, &p);
  if (st != MF_OK) return st;
  const bool dual = a.dyd != nullptr, norm = a.gq != nullptr;
  if (!both(a.dyd, a.dxd) || (a.gqd && !dual)) return MF_ERR_INVALID_ARG;
  if (norm && (!a.dgq || !a.dgk || (dual && (!a.dgqd || !a.dgkd || !a.xd)) || !a.work ||
               !aligned(a.work) || a.work_bytes < rope_work(a, dual)))
    return MF_ERR_INVALID_ARG;
  if (a.n_rows == 0) {   // sums over no rows
    cudaError_t e = cudaSuccess;
    if (norm)
      for (float* g : {a.dgq, a.dgk, a.dgqd, a.dgkd})
        if (g && e == cudaSuccess)
          e = cudaMemsetAsync(g, 0, sizeof(float) * a.head_dim, static_cast<cudaStream_t>(stream));
    return done(e);
  }
  const int64_t cols = static_cast<int64_t>(a.n_heads + a.n_kv_heads + a.n_copy_heads) * a.head_dim;
  const int64_t qk = static_cast<int64_t>(a.n_heads + a.n_kv_heads) * a.head_dim;
  if (!rows_ok(a.dy, a.lddy, cols, a.n_rows) || !rows_ok(a.dx, a.lddx, cols, a.n_rows) ||
      !aligned(a.dyd) || !aligned(a.dxd) || !in_place_ok(a.dy, a.lddy, a.dx, a.lddx, true) ||
      (dual && !in_place_ok(a.dyd, a.lddy, a.dxd, a.lddx, true)) ||
      (norm && (!rows_ok(a.x, a.ldx, qk, a.n_rows) || (dual && !aligned(a.xd)))))
    return MF_ERR_INVALID_ARG;
  // a warp has read all of its part of a row before it writes any: dx may be x too
  const bool over_x = in_place_ok(a.x, a.ldx, a.dx, a.lddx, a.x_prec == a.y_prec) &&
                      (!dual || in_place_ok(a.xd, a.ldx, a.dxd, a.lddx, a.x_prec == a.y_prec));
  if ((norm && !over_x) ||
      !outputs_apart({a.dx, a.dxd, a.dgq, a.dgk, a.dgqd, a.dgkd, norm ? a.work : nullptr},
                     {a.dx == a.dy ? nullptr : a.dy, a.dxd == a.dyd ? nullptr : a.dyd,
                      !norm || a.dx == a.x ? nullptr : a.x, !norm || a.dxd == a.xd ? nullptr : a.xd, a.gq,
                      a.gk, a.gqd, a.gkd}))
    return MF_ERR_INVALID_ARG;
  p.dy = a.dy; p.dyd = a.dyd; p.lddy = a.lddy;
  p.dx = a.dx; p.dxd = a.dxd; p.lddx = a.lddx;
  p.dgq = a.dgq; p.dgk = a.dgk; p.dgqd = a.dgqd; p.dgkd = a.dgkd;
  p.part = static_cast<float*>(a.work);
  return done(mf::qk_rope(p, true, a.x_prec == MF_PREC_BF16, a.y_prec == MF_PREC_BF16,
                          static_cast<cudaStream_t>(stream)));
}

mf_status mf_attn_work_bytes(const mf_attn_args* args, size_t* bytes) {
  if (!args || !bytes || args->n_rows < 0 || args->n_rows > INT32_MAX - 256 || args->n_heads < 1 ||
      args->n_heads > 65536)
    return MF_ERR_INVALID_ARG;
  *bytes = attn_work(*args);
  return MF_OK;
}

mf_status mf_attn_fwd(const mf_attn_args* args, void* stream) {
  if (!args) return MF_ERR_INVALID_ARG;
  AttnParams p;
  const mf_status st = attn_params(*args, false, &p, 0);
  if (st != MF_OK || args->n_rows == 0) return st;
  return done(mf::attn_tc_fwd(p, args->qd != nullptr, static_cast<cudaStream_t>(stream)));
}

mf_status mf_attn_bwd(const mf_attn_args* args, void* stream) {
  if (!args) return MF_ERR_INVALID_ARG;
  AttnParams p;
  const mf_status st = attn_params(*args, true, &p, attn_work(*args));
  if (st != MF_OK || args->n_rows == 0) return st;
  return done(mf::attn_tc_bwd(p, args->qd != nullptr, static_cast<cudaStream_t>(stream)));
}

mf_status mf_attn_window_work_bytes(const mf_attn_args* args, int64_t window, int n_sink, size_t* bytes) {
  if (!args || !bytes || args->n_rows < 0 || args->n_rows > INT32_MAX - 256 ||
      !heads_ok(args->n_heads, args->n_kv_heads, 0, args->head_dim) || window < 1 || n_sink < 0)
    return MF_ERR_INVALID_ARG;
  if (n_sink > mf::kMaxSinks) return MF_ERR_UNSUPPORTED;
  *bytes = window_work(*args, window, n_sink);
  return MF_OK;
}

mf_status mf_attn_window_fwd(const mf_attn_args* args, int64_t window, int n_sink, void* stream) {
  return attn_window(args, window, n_sink, false, stream);
}

mf_status mf_attn_window_bwd(const mf_attn_args* args, int64_t window, int n_sink, void* stream) {
  return attn_window(args, window, n_sink, true, stream);
}

mf_status mf_embed_work_bytes(const mf_embed_args* args, size_t* bytes) {
  if (!args || !bytes || !embed_sizes_ok(*args)) return MF_ERR_INVALID_ARG;
  *bytes = embed_work(*args);
  return MF_OK;
}

mf_status mf_embed_fwd(const mf_embed_args* args, void* stream) {
  if (!args) return MF_ERR_INVALID_ARG;
  const mf_embed_args& a = *args;
  EmbedParams p;
  const mf_status st = embed_params(a, &p);
  if (st != MF_OK) return st;
  if (!prec_ok(a.e_prec)) return MF_ERR_INVALID_ARG;
  if (a.n_rows == 0) return MF_OK;
  if (!both(a.Ed, a.yd) || !rows_ok(a.E, a.ldE, a.dim, a.vocab) || !rows_ok(a.y, a.ldy, a.dim, a.n_rows) || !aligned(a.Ed) ||
      !aligned(a.yd) || !outputs_apart({a.y, a.yd}, {a.E, a.Ed, a.ids}))
    return MF_ERR_INVALID_ARG;
  p.E = a.E; p.Ed = a.Ed; p.ldE = a.ldE;
  p.y = a.y; p.yd = a.yd; p.ldy = a.ldy;
  return done(mf::embed_fwd(p, a.e_prec == MF_PREC_BF16, a.y_prec == MF_PREC_BF16, static_cast<cudaStream_t>(stream)));
}

mf_status mf_embed_bwd(const mf_embed_args* args, void* stream) {
  if (!args) return MF_ERR_INVALID_ARG;
  const mf_embed_args& a = *args;
  EmbedParams p;
  const mf_status st = embed_params(a, &p);
  if (st != MF_OK) return st;
  if ((a.n_rows > 0 && !both(a.dyd, a.dEd)) || !rows_ok(a.dE, a.lddE, a.dim, a.vocab) || !aligned(a.dEd) ||
      (a.n_rows > 0 && (!rows_ok(a.dy, a.lddy, a.dim, a.n_rows) || !aligned(a.dyd))) || !a.work || !aligned(a.work) ||
      a.work_bytes < embed_work(a) ||
      !outputs_apart({a.dE, a.dEd, a.work}, {a.dy, a.dyd, a.ids}))
    return MF_ERR_INVALID_ARG;
  p.dy = a.dy; p.dyd = a.dyd; p.lddy = a.lddy;
  p.dE = a.dE; p.dEd = a.dEd; p.lddE = a.lddE;
  return done(mf::embed_bwd(p, a.y_prec == MF_PREC_BF16, a.work, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
