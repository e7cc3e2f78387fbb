// eql_encoder_api.cpp -- the C ABI declared in include/eqlinear_encoder.h: argument
// checks, plans and dispatch.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/eqlinear_encoder.h"
#include "eql_attn_args.h"
#include "eql_check.h"
#include "eql_encoder.h"
#include "eql_launch.h"

using eqk::align256;
using eqk::aligned;
using eqk::any_overlap;
using eqk::check_device;
using eqk::elem_bytes;
using eqk::overlaps;
using eqk::Range;
using eqk::valid_dtype;

namespace {

int launched(hipError_t e) { return e == hipSuccess ? EQL_OK : EQL_ERR_LAUNCH; }

constexpr int64_t kMaxElems = (int64_t)1 << 46;  // of any tensor, strides included

// Bytes from the first to the last element of [n0, n1, n2, inner] with these
// strides; 0 if a dimension is empty, -1 if a stride is negative or the span too large.
int64_t span(int64_t n0, int64_t n1, int64_t n2, int64_t inner, const int64_t* st, size_t e) {
  if (n0 == 0 || n1 == 0 || n2 == 0) return 0;
  const int64_t n[3] = {n0, n1, n2};
  int64_t s = inner;
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return -1;
    if (n[i] > 1 && st[i] > kMaxElems / n[i]) return -1;
    s += (n[i] - 1) * st[i];
  }
  return s > kMaxElems ? -1 : s * (int64_t)e;
}

// Whether no two elements of [n0, n1, n2, inner] share a place: every stride at least what
// the smaller ones span.  An output that is written twice would depend on the order.
bool distinct(int64_t n0, int64_t n1, int64_t n2, int64_t inner, const int64_t* st) {
  const int64_t n[3] = {n0, n1, n2};
  bool done[3] = {n0 <= 1, n1 <= 1, n2 <= 1};
  int64_t extent = inner;
  for (int i = 0; i < 3; ++i) {
    int at = -1;
    for (int k = 0; k < 3; ++k)
      if (!done[k] && (at < 0 || st[k] < st[at])) at = k;
    if (at < 0) break;
    if (st[at] < extent) return false;
    extent += (n[at] - 1) * st[at];
    done[at] = true;
  }
  return true;
}

// One axis of two outputs with the same stride.
struct Axis {
  int64_t na, nb, stride;
};
// Whether some element of an output (`inner` elements at every step of its axes) lies on one of
// another, whose first element is `delta` elements behind.  Axes from the largest stride
// on: only displacements at which what the smaller ones span could meet are looked at, two or
// three where elements lie apart (more than 64 count as meeting).
bool meet(const Axis* ax, int n, int64_t delta, int64_t inner) {
  if (n == 0) return delta < inner && delta > -inner;
  int64_t ea = inner, eb = inner;
  for (int i = 1; i < n; ++i) {
    ea += (ax[i].na - 1) * ax[i].stride;
    eb += (ax[i].nb - 1) * ax[i].stride;
  }
  auto floor_div = [](int64_t a, int64_t b) { return a / b - (a % b < 0); };
  const int64_t s = ax[0].stride;
  int64_t lo = floor_div(-eb - delta, s) + 1, hi = -floor_div(delta - ea, s) - 1;  // -eb < delta + d s < ea
  if (lo < 1 - ax[0].na) lo = 1 - ax[0].na;
  if (hi > ax[0].nb - 1) hi = ax[0].nb - 1;
  if (hi - lo >= 64) return true;
  for (int64_t d = lo; d <= hi; ++d)
    if (meet(ax + 1, n - 1, delta + d * s, inner)) return true;
  return false;
}

}  // namespace

namespace eqk {

// Key tiles that a workgroup of `rows` packed rows may walk.
static int64_t attn_tiles(const AttnArgs& a, int64_t tk, int64_t rows) {
  int64_t keys = (int64_t)a.left + a.right + (rows + a.G - 1) / a.G + a.sinks + 2 * tk;
  if (keys > a.Lk) keys = a.Lk;
  return (keys + tk - 1) / tk;
}

AttnPlan attn_plan(const AttnArgs& a, int dt, int cus) {
  AttnPlan p;
  // Up to 32 rows the waves of a workgroup share the rows and split the keys (a wave has no
  // registers for that with wide heads in full precision).
  p.waves = a.R <= 32 && (dt != kF32 || a.D <= 64) ? 1 : 4;
  const int64_t rows = 32 * p.waves;
  const int64_t blocks = (int64_t)a.B * a.Hkv * ((a.R + rows - 1) / rows);
  // workgroups that fill the device, and the tiles that are worth a part and its join: eight of
  // each of four waves, or two of a workgroup that shares its tiles
  const int64_t want = (p.waves == 1 ? 8 : 2) * (int64_t)cus, least = p.waves == 1 ? 32 : 2;
  int64_t parts = 1;
  if (blocks * 2 <= want) {
    const int64_t most = attn_tiles(a, attn_fwd_tile(dt, p.waves), rows) / least;
    parts = want / blocks;
    if (parts > most) parts = most;
    if (parts > 64) parts = 64;
    if (parts < 1) parts = 1;
  }
  p.parts = (int)parts;
  return p;
}

size_t attn_part_bytes(const AttnArgs& a, const AttnPlan& p) {
  return p.parts > 1 ? align256((size_t)a.B * a.Hkv * a.R * p.parts * (a.D + 2) * sizeof(float)) : 0;
}

size_t attn_dkv_plan(AttnArgs& a, int dt, int cus) {
  const int64_t tq = attn_tile(dt);
  const int64_t kt = ((int64_t)a.Lk + kAttnDkvKeys - 1) / kAttnDkvKeys;
  const int64_t all = ((int64_t)a.R + tq - 1) / tq;  // row tiles of the longest run
  int64_t run = ((int64_t)a.left + a.right + kAttnDkvKeys) * a.G / tq + 2;
  if (run > all) run = all;
  a.key_tiles = (int)kt;
  // key tiles with first tokens, where their run is longer than the others'
  int64_t st = run < all ? ((int64_t)a.sinks + kAttnDkvKeys - 1) / kAttnDkvKeys : 0;
  if (st > kt) st = kt;
  a.sink_tiles = (int)st;
  // the others are split only to fill the device
  const int64_t blocks = (int64_t)a.B * a.Hkv * kt;
  int64_t parts = 1;
  if (blocks > 0 && blocks * 2 <= cus) {  // (no keys: no blocks)
    parts = cus / blocks;
    if (parts > run / 4) parts = run / 4;
    if (parts > 32) parts = 32;
    if (parts < 1) parts = 1;
  }
  a.key_parts = (int)parts;
  a.run_tiles = (int)(run > 1 ? run : 1);
  // the first ones down to the others' length, but to no more than 8 parts a CU in all: enough to even
  // out the work, and what the parts take of memory does not grow with the shape (768 head pairs of
  // 2,048 tokens, 4 first ones: two parts 1.34 ms, eleven 1.30; 16 pairs of 16,384 with 300: 243 us, 288)
  int64_t sp = st ? (all * parts + run - 1) / run : 1;
  const int64_t most = st ? 8 * (int64_t)cus / ((int64_t)a.B * a.Hkv * st) : 1;
  if (sp > most) sp = most;
  if (sp > 128) sp = 128;
  if (sp < 1) sp = 1;
  a.sink_parts = (int)sp;
  const int64_t slots = (sp > 1 ? st * sp : 0) + (parts > 1 ? (kt - st) * parts : 0);
  return align256((size_t)a.B * a.Hkv * slots * 2 * kAttnDkvKeys * a.D * sizeof(float));
}

}  // namespace eqk

namespace {

// Checks the shape and fills the arguments that do not hold addresses.
int window_args(const eqlinear_window_shape* s, eqk::AttnArgs& a) {
  if (!s || !valid_dtype(s->dtype) || s->B < 0 || s->Lq < 0 || s->Lk < 0 || s->heads < 1 || s->kv_heads < 1 ||
      s->head_dim < 1 || s->heads % s->kv_heads != 0 || s->left < -1 || s->right < -1 || s->sinks < 0 ||
      !(s->scale > 0.0f) || isinf(s->scale) || s->reserved != 0)
    return EQL_ERR_INVALID_ARG;
  const int64_t g = s->heads / s->kv_heads;
  const size_t e = elem_bytes(s->dtype);
  if (s->B > (1 << 24) || s->Lk > eqk::kAttnMaxPos || s->heads > 65536 || s->Lq >= ((int64_t)1 << 29) / g ||
      s->head_dim > eqk::kAttnMaxD || (size_t)s->head_dim * e % 16 != 0)
    return EQL_ERR_UNSUPPORTED;
  // one launch's grid holds at least one sequence: 2^20 tiles, what rounding their number to whole
  // runs adds (2^20 at most), and the parts (8 a CU at most) are well below 2^32 threads
  if (s->kv_heads * ((s->Lq * g + 31) / 32) >= ((int64_t)1 << 20) ||
      s->kv_heads * ((s->Lk + eqk::kAttnDkvKeys - 1) / eqk::kAttnDkvKeys) >= ((int64_t)1 << 20))
    return EQL_ERR_UNSUPPORTED;
  auto lim = [](int64_t v) { return v < 0 || v > eqk::kAttnNoLimit ? eqk::kAttnNoLimit : (int)v; };
  a = eqk::AttnArgs{};
  a.B = (int)s->B;
  a.Lq = (int)s->Lq;
  a.Lk = (int)s->Lk;
  a.Hkv = s->kv_heads;
  a.G = (int)g;
  a.R = (int)(s->Lq * g);
  a.D = s->head_dim;
  a.left = lim(s->left);
  a.right = lim(s->right);
  a.sinks = (int)(s->sinks > s->Lk ? s->Lk : s->sinks);
  a.scale = s->scale;
  a.scale_log2e = (float)(s->scale * 1.4426950408889634);
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = s->q_stride[i];
    a.ks[i] = s->k_stride[i];
    a.vs[i] = s->v_stride[i];
    a.os[i] = s->o_stride[i];
    a.gos[i] = s->do_stride[i];
    a.dqs[i] = s->dq_stride[i];
    a.dks[i] = s->dk_stride[i];
    a.dvs[i] = s->dv_stride[i];
  }
  return EQL_OK;
}

// One tensor of the attention, and one buffer without strides.
struct Operand {
  const void* p;
  const int64_t* st;
  bool query, written;
};
struct Buffer {
  Range r;
  bool written;
};

// Whether two outputs whose spans overlap share a place.  Their strides have to agree (on
// axes where both take a step) for them to lie between one another's elements.
bool outputs_meet(const eqlinear_window_shape* s, const Operand& x, const Operand& y) {
  const int64_t nx[3] = {s->B, x.query ? s->Lq : s->Lk, x.query ? s->heads : s->kv_heads};
  const int64_t ny[3] = {s->B, y.query ? s->Lq : s->Lk, y.query ? s->heads : s->kv_heads};
  const int64_t e = (int64_t)elem_bytes(s->dtype);
  Axis ax[3];
  int n = 0;
  for (int i = 0; i < 3; ++i) {
    if (nx[i] == 1 && ny[i] == 1) continue;
    if (nx[i] > 1 && ny[i] > 1 && x.st[i] != y.st[i]) return true;
    const Axis a{nx[i], ny[i], nx[i] > 1 ? x.st[i] : y.st[i]};
    int at = n++;
    for (; at > 0 && ax[at - 1].stride < a.stride; --at) ax[at] = ax[at - 1];
    ax[at] = a;
  }
  return meet(ax, n, ((intptr_t)y.p - (intptr_t)x.p) / e, s->head_dim);
}

int window_operands(const eqlinear_window_shape* s, const Operand* t, int n, const Buffer* buf, int nbuf) {
  const size_t e = elem_bytes(s->dtype);
  const int64_t ce = (int64_t)(16 / e);
  Range r[8];
  for (int i = 0; i < n; ++i) {
    const int64_t L = t[i].query ? s->Lq : s->Lk;
    const int64_t b = span(s->B, L, t[i].query ? s->heads : s->kv_heads, s->head_dim, t[i].st, e);
    if (b < 0) return EQL_ERR_INVALID_ARG;
    if (b > 0 && !t[i].p) return EQL_ERR_INVALID_ARG;
    if (b > 0 && t[i].written && !distinct(s->B, L, t[i].query ? s->heads : s->kv_heads, s->head_dim, t[i].st))
      return EQL_ERR_INVALID_ARG;
    for (int k = 0; k < 3; ++k)
      if (t[i].st[k] % ce != 0) return EQL_ERR_ALIGNMENT;
    // a tile's rows are addressed by 31 bits from its first: 64 tokens and the heads
    if ((double)(65 * (double)t[i].st[1] + (double)(t[i].query ? s->heads : 0) * (double)t[i].st[2]) * e >= 2147483648.0)
      return EQL_ERR_UNSUPPORTED;
    if (!aligned(t[i].p, 16)) return EQL_ERR_ALIGNMENT;
    r[i] = Range{t[i].p, (size_t)b};
  }
  // nothing that is written overlaps anything else; strided outputs may interleave in one buffer
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < n; ++j)
      if (t[i].written && j != i && overlaps(r[i], r[j]) && (!t[j].written || (j < i && outputs_meet(s, t[i], t[j]))))
        return EQL_ERR_INVALID_ARG;
    for (int j = 0; j < nbuf; ++j)
      if ((t[i].written || buf[j].written) && overlaps(r[i], buf[j].r)) return EQL_ERR_INVALID_ARG;
  }
  for (int i = 0; i < nbuf; ++i)
    for (int j = 0; j < i; ++j)
      if ((buf[i].written || buf[j].written) && overlaps(buf[i].r, buf[j].r)) return EQL_ERR_INVALID_ARG;
  return EQL_OK;
}

// Plans are made for this many CUs whatever the device, so that a workspace
// query and the call agree and results do not depend on the device.
constexpr int kPlanCus = 256;

size_t lse_bytes(const eqk::AttnArgs& a) { return (size_t)a.B * a.Hkv * a.R * sizeof(float); }
size_t delta_bytes(const eqk::AttnArgs& a) { return align256(lse_bytes(a)); }

}  // namespace

extern "C" {

int eqlinear_rotary(const eqlinear_rotary_shape* s, const void* x, const void* positions, const float* freqs, void* y,
                    void* stream) {
  if (!s || !valid_dtype(s->dtype) || s->B < 0 || s->L < 0 || s->heads < 1 || s->dh < 1 || s->T < 1 || s->axes < 1)
    return EQL_ERR_INVALID_ARG;
  if (s->axes > eqk::kRotaryMaxAxes || s->T > EQLINEAR_MAX_T || s->dh > eqk::kRotaryMaxDim ||
      (int64_t)s->dh * s->T > eqk::kRotaryMaxDim || s->heads > 65536 || s->B > ((int64_t)1 << 31) ||
      s->L > ((int64_t)1 << 31))
    return EQL_ERR_UNSUPPORTED;
  eqk::RotaryArgs a{};
  int64_t n = 0;
  for (int i = 0; i < s->axes; ++i) {
    if (s->sections[i] < 0 || s->sections[i] > s->dh) return EQL_ERR_INVALID_ARG;
    n += s->sections[i];
    a.ends[i] = (int)n;
  }
  for (int i = s->axes; i < eqk::kRotaryMaxAxes; ++i) a.ends[i] = (int)n;
  if (n < 1 || 2 * n > s->dh) return EQL_ERR_INVALID_ARG;
  const size_t e = elem_bytes(s->dtype);
  const int64_t D = (int64_t)s->dh * s->T;
  const int64_t xb = span(s->B, s->L, s->heads, D, s->x_stride, e), yb = span(s->B, s->L, s->heads, D, s->y_stride, e);
  const int64_t pst[3] = {s->pos_stride[0], s->pos_stride[1], 0};
  const int64_t pb = span(s->B, s->L, 1, s->axes, pst, 4);
  if (xb < 0 || yb < 0 || pb < 0 || !freqs || (xb > 0 && (!x || !y || !positions))) return EQL_ERR_INVALID_ARG;
  if (yb > 0 && !distinct(s->B, s->L, s->heads, D, s->y_stride)) return EQL_ERR_INVALID_ARG;
  if (!aligned(x, e) || !aligned(y, e) || !aligned(positions, 4) || !aligned(freqs, 4)) return EQL_ERR_ALIGNMENT;
  bool in_place = x == y;
  for (int i = 0; i < 3; ++i) in_place = in_place && s->x_stride[i] == s->y_stride[i];
  const Range ry{y, (size_t)yb};
  if ((!in_place && overlaps(ry, Range{x, (size_t)xb})) || overlaps(ry, Range{positions, (size_t)pb}) ||
      overlaps(ry, Range{freqs, (size_t)n * 4}))
    return EQL_ERR_INVALID_ARG;
  if (int st = check_device()) return st;
  if (xb == 0) return EQL_OK;
  a.x = x;
  a.y = y;
  a.positions = positions;
  a.freqs = freqs;
  a.tokens = s->B * s->L;
  a.L = s->L;
  a.N = s->heads;
  a.T = s->T;
  a.n = (int)n;
  a.D = (int)D;
  a.float_pos = s->float_positions != 0;
  a.interleaved = s->interleaved != 0;
  a.copy_rest = !in_place;
  a.sign = s->inverse ? -1.0f : 1.0f;
  a.ps[0] = s->pos_stride[0];
  a.ps[1] = s->pos_stride[1];
  // elements a thread takes at once: the widest vector that divides every
  // run, stride and address
  int vec = (int)(16 / e);
  for (int i = 0; i < 3; ++i) {
    a.xs[i] = s->x_stride[i];
    a.ys[i] = s->y_stride[i];
    while (a.xs[i] % vec || a.ys[i] % vec) vec /= 2;
  }
  const int64_t run = !a.interleaved ? n * a.T : a.T > 1 ? a.T : 2 * n;
  while (run % vec || (2 * n * a.T) % vec || D % vec || (uintptr_t)x % (vec * e) || (uintptr_t)y % (vec * e)) vec /= 2;
  // tokens of a workgroup: about 1024 vectors, and the angles that fit
  const int64_t per = (a.N * (D / vec) + 1) / 2;
  int64_t tb = (1024 + per - 1) / per;
  if (tb * n > eqk::kRotaryAngles) tb = eqk::kRotaryAngles / n;
  if (tb > eqk::kRotaryMaxTokens) tb = eqk::kRotaryMaxTokens;
  a.TB = (int)(tb < 1 ? 1 : tb);
  return launched(eqk::launch_rotary(s->dtype, a, vec, (hipStream_t)stream));
}

size_t eqlinear_window_attention_workspace_bytes(const eqlinear_window_shape* s) {
  eqk::AttnArgs a;
  if (window_args(s, a) || a.B == 0 || a.R == 0) return 0;
  return eqk::attn_part_bytes(a, eqk::attn_plan(a, s->dtype, kPlanCus));
}

int eqlinear_window_attention(const eqlinear_window_shape* s, const void* q, const void* k, const void* v,
                              const int32_t* lengths, const int32_t* starts, void* o, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream) {
  eqk::AttnArgs a;
  if (int st = window_args(s, a)) return st;
  const Operand t[4] = {{q, a.qs, true, false}, {k, a.ks, false, false}, {v, a.vs, false, false}, {o, a.os, true, true}};
  if (!aligned(lengths, 4) || !aligned(starts, 4) || !aligned(lse, 4) || !aligned(workspace, 16)) return EQL_ERR_ALIGNMENT;
  const bool empty = a.B == 0 || a.R == 0;
  const eqk::AttnPlan p = empty ? eqk::AttnPlan{} : eqk::attn_plan(a, s->dtype, kPlanCus);
  const size_t need = empty ? 0 : eqk::attn_part_bytes(a, p);
  const Buffer buf[4] = {{{lengths, a.B * sizeof(int32_t)}, false}, {{starts, a.B * sizeof(int32_t)}, false},
                         {{lse, lse_bytes(a)}, true}, {{workspace, workspace_bytes < need ? workspace_bytes : need}, true}};
  if (int st = window_operands(s, t, 4, buf, 4)) return st;
  if (empty) return check_device();
  if (need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lengths = lengths;
  a.starts = starts;
  a.lse = lse;
  a.part = (float*)workspace;
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::wattn_fwd<eqk::kF32>(a, p, st));
  if (s->dtype == EQL_F16) return launched(eqk::wattn_fwd<eqk::kF16>(a, p, st));
  return launched(eqk::wattn_fwd<eqk::kBF16>(a, p, st));
}

size_t eqlinear_window_attention_backward_workspace_bytes(const eqlinear_window_shape* s) {
  eqk::AttnArgs a;
  if (window_args(s, a) || a.B == 0) return 0;
  return delta_bytes(a) + eqk::attn_dkv_plan(a, s->dtype, kPlanCus);
}

int eqlinear_window_attention_backward(const eqlinear_window_shape* s, const void* q, const void* k, const void* v,
                                       const int32_t* lengths, const int32_t* starts, const void* o, const float* lse,
                                       const void* d_o, void* dq, void* dk, void* dv, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  eqk::AttnArgs a;
  if (int st = window_args(s, a)) return st;
  const Operand t[8] = {{q, a.qs, true, false},  {k, a.ks, false, false},   {v, a.vs, false, false},
                        {o, a.os, true, false},  {d_o, a.gos, true, false}, {dq, a.dqs, true, true},
                        {dk, a.dks, false, true}, {dv, a.dvs, false, true}};
  if (!aligned(lengths, 4) || !aligned(starts, 4) || !aligned(lse, 4) || !aligned(workspace, 16)) return EQL_ERR_ALIGNMENT;
  const bool empty = a.B == 0 || (a.R == 0 && a.Lk == 0);
  const size_t part = empty ? 0 : eqk::attn_dkv_plan(a, s->dtype, kPlanCus), head = delta_bytes(a), need = head + part;
  const Buffer buf[4] = {{{lengths, a.B * sizeof(int32_t)}, false}, {{starts, a.B * sizeof(int32_t)}, false},
                         {{lse, lse_bytes(a)}, false}, {{workspace, workspace_bytes < need ? workspace_bytes : need}, true}};
  if (int st = window_operands(s, t, 8, buf, 4)) return st;
  if (empty) return check_device();
  if (a.R > 0 && !lse) return EQL_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = const_cast<void*>(o);
  a.go = d_o;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.lengths = lengths;
  a.starts = starts;
  a.lse = const_cast<float*>(lse);
  a.delta = (float*)workspace;
  a.part = part ? (float*)((char*)workspace + head) : nullptr;
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::wattn_bwd<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::wattn_bwd<eqk::kF16>(a, st));
  return launched(eqk::wattn_bwd<eqk::kBF16>(a, st));
}

}  // extern "C"

namespace {

int gn_args(int64_t B, int64_t S, int T, int C, int groups, int dtype, eqk::GnArgs& a) {
  if (!valid_dtype(dtype) || B < 0 || S < 0 || T < 1 || C < 1 || groups < 1 || C % groups != 0) return EQL_ERR_INVALID_ARG;
  if (T > EQLINEAR_MAX_T || C > 65536 || groups > eqk::kGnMaxGroups || B > (1 << 20) || S > ((int64_t)1 << 30))
    return EQL_ERR_UNSUPPORTED;
  if ((double)B * (double)S * C * T > (double)kMaxElems) return EQL_ERR_UNSUPPORTED;
  a = eqk::GnArgs{};
  a.B = B;
  a.S = S;
  a.C = C;
  a.T = T;
  a.G = groups;
  a.K = C * T;
  return EQL_OK;
}

// Whether every output is apart from the inputs and the other outputs.
bool apart(const Range* out, int n, const Range* in, int nin) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < nin; ++j)
      if (overlaps(out[i], in[j])) return false;
  return !any_overlap(out, n);
}

// Whole 16-byte vectors where every row starts on one.
int gn_vec(const eqk::GnArgs& a, int dtype) {
  const int w = (int)(16 / elem_bytes(dtype));
  return a.K % w == 0 ? w : 1;
}

}  // namespace

extern "C" {

size_t eqlinear_group_norm_act_workspace_bytes(int64_t B, int64_t S, int T, int C, int groups, int dtype) {
  eqk::GnArgs a;
  if (gn_args(B, S, T, C, groups, dtype, a) || B == 0 || S == 0) return 0;
  eqk::gn_plan(a, gn_vec(a, dtype), kPlanCus, false);
  return a.hold ? 0 : align256((size_t)B * a.chunks * a.cblocks * groups * 2 * sizeof(float));
}

int eqlinear_group_norm_act(const void* x, const void* weight, const void* bias, void* y, float* stats,
                            void* workspace, size_t workspace_bytes, int64_t B, int64_t S, int T, int C, int groups,
                            float eps, int act, int dtype, void* stream) {
  eqk::GnArgs a;
  if (int st = gn_args(B, S, T, C, groups, dtype, a)) return st;
  if (act < EQL_ACT_NONE || act > EQL_ACT_GELU || !(eps >= 0.0f) || !weight || !bias) return EQL_ERR_INVALID_ARG;
  const bool empty = B == 0 || S == 0;
  if (!empty && (!x || !y)) return EQL_ERR_INVALID_ARG;
  const size_t e = elem_bytes(dtype), n = (size_t)B * S * a.K * e;
  if (!aligned(x, 16) || !aligned(y, 16) || !aligned(weight, e) || !aligned(bias, e) || !aligned(stats, 8) ||
      !aligned(workspace, 16))
    return EQL_ERR_ALIGNMENT;
  const size_t need = eqlinear_group_norm_act_workspace_bytes(B, S, T, C, groups, dtype);
  const Range out[3] = {{y, n}, {stats, (size_t)B * groups * 8}, {workspace, workspace_bytes < need ? workspace_bytes : need}}, in[3] = {{x, n}, {weight, C * e}, {bias, C * e}};
  if (!apart(out, 3, in, 3)) return EQL_ERR_INVALID_ARG;
  if (empty) return check_device();
  const int vec = gn_vec(a, dtype);
  eqk::gn_plan(a, vec, kPlanCus, false);
  if (need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.x = x;
  a.w = weight;
  a.b = bias;
  a.y = y;
  a.stats = stats;
  a.part = (float*)workspace;
  a.eps = eps;
  a.act = act;
  return launched(eqk::launch_gn_forward(dtype, a, vec, (hipStream_t)stream));
}

size_t eqlinear_group_norm_act_backward_workspace_bytes(int64_t B, int64_t S, int T, int C, int groups, int dtype) {
  eqk::GnArgs a;
  if (gn_args(B, S, T, C, groups, dtype, a) || B == 0 || S == 0) return 0;
  eqk::gn_plan(a, gn_vec(a, dtype), kPlanCus, true);
  return (a.hold ? 0 : align256((size_t)B * a.chunks * C * 2 * sizeof(float))) + align256((size_t)B * C * 2 * sizeof(float));
}

int eqlinear_group_norm_act_backward(const void* x, const void* weight, const void* bias, const float* stats,
                                     const void* dy, void* dx, void* dw, void* db, void* workspace,
                                     size_t workspace_bytes, int64_t B, int64_t S, int T, int C, int groups, int act,
                                     int dtype, void* stream) {
  eqk::GnArgs a;
  if (int st = gn_args(B, S, T, C, groups, dtype, a)) return st;
  if (act < EQL_ACT_NONE || act > EQL_ACT_GELU || !weight || !bias) return EQL_ERR_INVALID_ARG;
  const bool empty = B == 0 || S == 0;
  if (!empty && (!x || !dy || !dx || !stats || !dw || !db)) return EQL_ERR_INVALID_ARG;
  const size_t e = elem_bytes(dtype), n = (size_t)B * S * a.K * e;
  if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(weight, e) || !aligned(bias, e) ||
      !aligned(dw, e) || !aligned(db, e) || !aligned(stats, 8) || !aligned(workspace, 16))
    return EQL_ERR_ALIGNMENT;
  const size_t need = eqlinear_group_norm_act_backward_workspace_bytes(B, S, T, C, groups, dtype);
  const Range out[4] = {{dx, n}, {dw, C * e}, {db, C * e}, {workspace, workspace_bytes < need ? workspace_bytes : need}};
  const Range in[5] = {{x, n}, {dy, n}, {weight, C * e}, {bias, C * e}, {stats, (size_t)B * groups * 8}};
  if (!apart(out, 4, in, 5)) return EQL_ERR_INVALID_ARG;
  if (empty) return check_device();
  const int vec = gn_vec(a, dtype);
  eqk::gn_plan(a, vec, kPlanCus, true);
  if (!workspace || workspace_bytes < need) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.x = x;
  a.w = weight;
  a.b = bias;
  a.dy = dy;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  a.stats = const_cast<float*>(stats);
  a.part = (float*)workspace;
  a.sums = (float*)((char*)workspace + (a.hold ? 0 : align256((size_t)B * a.chunks * C * 2 * sizeof(float))));
  a.act = act;
  return launched(eqk::launch_gn_backward(dtype, a, vec, (hipStream_t)stream));
}

}  // extern "C"
