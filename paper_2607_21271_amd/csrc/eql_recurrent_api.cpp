// eql_recurrent_api.cpp -- the C ABI declared in include/eqlinear_recurrent.h: argument
// checks, plans and dispatch.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/eqlinear_encoder.h"
#include "../../include/eqlinear_recurrent.h"
#include "eql_check.h"
#include "eql_recurrent.h"

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
constexpr int64_t kMaxB = (int64_t)1 << 20, kMaxL = (int64_t)1 << 30;
constexpr int kMaxCols = 65536;
// Plans are made for this many CUs whatever the device, so that a workspace
// query and the call agree and results do not depend on the device.
constexpr int kPlanCus = 256;

// Bytes from the first to the last element of [n0, n1, n2, inner] with these strides; 0
// if a dimension is empty, -1 if a stride is negative or the span too large.
int64_t span(int64_t n0, int64_t n1, int64_t n2, int64_t inner, const int64_t* st, size_t e) {
  if (n0 == 0 || n1 == 0 || n2 == 0 || inner == 0) return 0;
  const int64_t n[3] = {n0, n1, n2};
  int64_t s = inner;
  for (int i = 0; i < 3; ++i) {
    if (i == 2 && n2 == 1) continue;
    if (st[i] < 0) return -1;
    if (n[i] > 1 && st[i] > kMaxElems / n[i]) return -1;
    s += (n[i] - 1) * st[i];
  }
  return s > kMaxElems ? -1 : s * (int64_t)e;
}

// Whether every output is apart from the inputs and the other outputs.
bool apart(const Range* out, int n, const Range* in, int nin) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < nin; ++j)
      if (overlaps(out[i], in[j])) return false;
  return !any_overlap(out, n);
}

// Whether a tensor with these strides and every row of `inner` elements can be read in vectors of `vec`.
bool vectors(const void* p, const int64_t* st, int n, size_t e, int vec) {
  if (!p) return true;
  for (int i = 0; i < n; ++i)
    if (st[i] % vec != 0) return false;
  return aligned(p, vec * e);
}

// ---- selective scan ----

int scan_args(const eqlinear_scan_shape* s, eqk::ScanArgs& a, bool bwd) {
  if (!s || !valid_dtype(s->dtype) || s->B < 0 || s->L < 0 || s->C < 1 || s->T < 1 || s->N < 1 || s->groups < 1 ||
      s->C % s->groups != 0 || s->softplus < 0 || s->softplus > 1)
    return EQL_ERR_INVALID_ARG;
  if (s->T > EQLINEAR_MAX_T || (int64_t)s->C * s->T > kMaxCols || s->N > eqk::kScanMaxN || s->B > kMaxB || s->L > kMaxL ||
      (double)s->B * (double)s->L * s->C * s->T > (double)kMaxElems || (double)s->B * s->C * s->T * s->N > (double)kMaxElems)
    return EQL_ERR_UNSUPPORTED;
  a = eqk::ScanArgs{};
  a.B = s->B;
  a.L = s->L;
  a.C = s->C;
  a.T = s->T;
  a.N = s->N;
  a.G = s->groups;
  a.softplus = s->softplus;
  for (int i = 0; i < 2; ++i) {
    a.xs[i] = s->x_stride[i];
    a.ds[i] = s->delta_stride[i];
    a.zs[i] = s->z_stride[i];
  }
  for (int i = 0; i < 3; ++i) {
    a.bs[i] = s->b_stride[i];
    a.cs[i] = s->c_stride[i];
  }
  eqk::scan_plan(a, kPlanCus, bwd);
  return EQL_OK;
}

int64_t scan_np(const eqk::ScanArgs& a) { return 4 * eqk::scan_lanes(a.N); }
size_t scan_states(const eqk::ScanArgs& a) { return (size_t)a.B * a.runs * a.cols * scan_np(a) * sizeof(float); }
size_t scan_carry(const eqk::ScanArgs& a) {
  return a.K > 1 ? align256((size_t)a.B * a.K * a.cols * scan_np(a) * sizeof(float)) : 0;
}
size_t scan_sums(const eqk::ScanArgs& a) { return a.K > 1 ? align256((size_t)a.B * a.K * a.cols * sizeof(float)) : 0; }
size_t scan_part(const eqk::ScanArgs& a) { return align256((size_t)a.B * a.K * (a.N + 2) * a.cols * sizeof(float)); }
size_t scan_bcpart(const eqk::ScanArgs& a) {
  return a.P > 1 ? align256((size_t)a.B * a.L * a.G * a.P * 2 * scan_np(a) * sizeof(float)) : 0;
}

// Spans of the inputs that both passes read; the status of their checks.
struct ScanInputs {
  Range r[9];
};
int scan_inputs(const eqlinear_scan_shape* s, const eqk::ScanArgs& a, const void* x, const void* delta, const float* A,
                const void* b, const void* c, const float* D, const void* z, const float* bias, const int32_t* lengths,
                ScanInputs& in) {
  const size_t e = elem_bytes(s->dtype);
  const bool empty = a.B == 0 || a.L == 0;
  const int64_t xst[3] = {a.xs[0], a.xs[1], 0}, dst[3] = {a.ds[0], a.ds[1], 0}, zst[3] = {a.zs[0], a.zs[1], 0};
  const int64_t bytes[9] = {span(a.B, a.L, 1, a.CT, xst, e),  span(a.B, a.L, 1, a.CT, dst, e),
                            (int64_t)a.C * a.N * 4,           span(a.B, a.L, a.G, a.N, a.bs, e),
                            span(a.B, a.L, a.G, a.N, a.cs, e), D ? (int64_t)a.C * 4 : 0,
                            z ? span(a.B, a.L, 1, a.CT, zst, e) : 0, bias ? (int64_t)a.C * 4 : 0,
                            lengths ? a.B * 4 : 0};
  const void* ptr[9] = {x, delta, A, b, c, D, z, bias, lengths};
  for (int i = 0; i < 9; ++i) {
    if (bytes[i] < 0) return EQL_ERR_INVALID_ARG;
    in.r[i] = Range{ptr[i], (size_t)bytes[i]};
  }
  if (!A || (!empty && (!x || !delta || !b || !c))) return EQL_ERR_INVALID_ARG;
  for (int i = 0; i < 9; ++i)
    if (!aligned(ptr[i], i == 2 || i == 5 || i >= 7 ? 4 : e)) return EQL_ERR_ALIGNMENT;
  return EQL_OK;
}

// How the kernels read and write: a tile's tokens are addressed by 31 bits from its first.
int scan_mode(const eqk::ScanArgs& a, int dtype) {
  const int NL = eqk::scan_lanes(a.N), vec = eqk::scan_vec(dtype, NL, eqk::scan_columns(NL));
  const int64_t steps[6] = {a.CT, a.xs[1], a.ds[1], a.z ? a.zs[1] : 0, a.bs[1], a.cs[1]};
  for (int64_t st : steps)
    if (st >= ((int64_t)1 << 31) / 128) return eqk::kTiny;
  if (a.CTg < vec) return eqk::kTiny;
  return a.CTg % vec == 0 && a.N % 4 == 0 && aligned(a.A, 16) ? eqk::kWhole : eqk::kLoose;
}

}  // namespace

namespace eqk {

// Microseconds of a kernel whose waves, w to a SIMD, walk `tokens` tokens each: its start, and for a token `each` a wave and
// `round` where `slots` of them hide the rest of each other's time.  Measured at 16 states: forward 0.19, 0.31 and 0.55 us a
// token with 1, 2 and 4 waves a SIMD, gradients 0.60, 0.90 and 1.80; above 32 states, with four columns a lane, 0.31 and 0.50
// and, gradients, 1.2 a wave.  The same rates are taken for fewer states, where tiles are of four or eight tokens (8,192
// tokens of 1,024 f16 columns of 1 and 4 states, the gradients' kernel: 53 and 51 us, of 7 states 84, of 16 114).
struct ScanRate {
  double start, round, each;
  int slots;
};
static double scan_time(int64_t waves, int64_t tokens, int64_t simds, const ScanRate& r) {
  const int64_t w = (waves + simds - 1) / simds;
  return r.start + (double)tokens * (r.round * (double)((w + r.slots - 1) / r.slots) + r.each * (double)w);
}

// Chunks of tokens where the columns alone do not fill the device: the number of waves (one to four a SIMD) for which the
// main pass and the one before it over states or gradients, 0.7 of the forward's main one, take least.
// Gradients: workgroups of four, two or one wave, which fill a CU's four SIMDs alike (three where there are no more); smaller
// ones leave fewer waves without columns, and more sums of db and dc to memory.
void scan_plan(ScanArgs& a, int cus, bool bwd) {
  const int NL = scan_lanes(a.N), CH = scan_cols(NL), TT = scan_tile(NL), back = scan_cols(NL, scan_columns(NL));
  a.CT = a.C * a.T;
  a.CTg = a.CT / a.G;
  a.nblk = (a.CTg + CH - 1) / CH;
  a.bblk = (a.CTg + back - 1) / back;
  a.cols = a.G * a.nblk * CH;
  a.tiles = (a.L + TT - 1) / TT;
  a.runs = (a.L + scan_run(NL) - 1) / scan_run(NL);
  a.mT = channel_factor(a.T);
  const int64_t simds = 4 * (int64_t)cus, tiles = a.tiles > 0 ? a.tiles : 1, first = a.B * a.G * a.bblk;
  const int nblk = a.bblk;
  const bool two = back < CH;
  const ScanRate forward = two ? ScanRate{7.0, 0.065, 0.122, 4} : ScanRate{7.0, 0.11, 0.195, 2};
  const ScanRate main = !bwd ? forward : two ? ScanRate{12.0, 0.3, 0.3, 2} : ScanRate{12.0, 0.0, 1.2, 1};
  int64_t per = tiles;
  double least = -1.0;
  for (int waves = nblk < kScanWaves ? nblk : kScanWaves; waves > 0; --waves) {
    if (waves == 3 && nblk > 3) continue;
    const int P = (nblk + waves - 1) / waves;
    const int64_t one = a.B * a.G * (bwd ? (int64_t)P * waves : nblk);
    // the sums' way out and back in, at 5 TB/s, and a launch
    const double sums = bwd && P > 1 ? (double)a.B * a.L * a.G * P * 16 * 4 * NL / 5e6 + 4.0 : 0.0;
    auto take = [&](int64_t n, double t) {
      if (least >= 0.0 && t + sums >= least) return;
      least = t + sums;
      per = n;
      a.P = P;
      a.waves = waves;
    };
    take(tiles, scan_time(one, tiles * TT, simds, main));
    for (int w = 1; w <= 4 && one > 0 && one < 2 * simds; ++w) {
      int64_t K = w * simds / one;
      if (K > tiles) K = tiles;
      if (K < 2) continue;
      const int64_t n = (tiles + K - 1) / K;
      K = (tiles + n - 1) / n;
      // two more launches, and the states between the passes: written, carried over the chunks and read
      const double carry = 7.0 + (double)(a.B * K) * a.cols * 4 * NL * 16 / 5e6;
      take(n, scan_time(one * K, n * TT, simds, main) + 0.7 * scan_time(first * K, n * TT, simds, forward) + carry);
    }
    if (!bwd) break;
  }
  a.chunk = per * TT;
  a.K = (int)((tiles + per - 1) / per);
}

void conv_plan(ConvArgs& a, int dt, int cus, bool bwd) {
  const int vec = conv_vec(dt, a.W, bwd);
  a.CT = a.C * a.T;
  a.mT = channel_factor(a.T);
  const int nv = (a.CT + vec - 1) / vec;
  a.width = nv < 256 ? nv : 256;
  a.cblocks = (nv + a.width - 1) / a.width;
  a.turns = 256 / a.width;
  a.rows = 16;
  if (bwd) {
    // strips of 8 m tokens with their halo: longer ones, which read less of it twice, where the device has two waves a
    // SIMD anyway
    int64_t m = a.B * nv * a.L / (8 * 64 * 8 * (int64_t)cus);
    m = m < 2 ? 2 : m > 8 ? 8 : m;
    a.rows = (int)(8 * m) - (a.W - 1);
  }
  a.strips = (a.L + a.rows - 1) / a.rows;
  if (a.strips < 1) a.strips = 1;
  a.groups = (a.strips + a.turns - 1) / a.turns;
}

void res_plan(ResArgs& a, int dt, int cus, bool bwd) {
  (void)dt;
  a.K = a.C * a.T;
  a.mT = channel_factor(a.T);
  // The fewest threads that hold a row in eight elements each: 32 MiB of f16 rows of 16 elements take 72 us with 4 threads
  // and 252 with 16, of 256 elements 46 us with 32 and 76 with 64.  Up to 4096 elements 16 each save barriers; above, 1024
  // threads of eight (512 of 16 spill in the backward: training passes over 8192 f16 columns 281 us instead of 395).
  a.lanes = a.K <= 256 ? 4 : a.K <= 1024 ? 64 : a.K <= 4096 ? 256 : 1024;
  while (8 * a.lanes < a.K && a.K <= 256) a.lanes *= 2;
  a.ept = a.K <= 8 * a.lanes ? 8 : 16;
  a.seqs = a.gate ? a.B : 1;
  a.rows = a.gate ? a.L : a.B * a.L;
  const int64_t turn = a.lanes < 256 ? 256 / a.lanes : 1;  // rows of a workgroup at a time
  // four workgroups a CU (two in the backward, whose sums take registers), each at least two turns long
  int64_t strips = a.seqs > 0 ? ((bwd ? 2 : 4) * (int64_t)cus + a.seqs - 1) / a.seqs : 1;
  const int64_t most = (a.rows + 2 * turn - 1) / (2 * turn);
  // gradients: no more than 256 turns, which a thread adds up one after the other
  const int64_t least = bwd ? (a.rows + 256 * turn - 1) / (256 * turn) : 1;
  if (strips < least) strips = least;
  if (strips > most) strips = most;
  if (strips < 1) strips = 1;
  a.strip = (a.rows + strips - 1) / strips;
  if (a.strip < 1) a.strip = 1;
  a.strips = a.rows > 0 ? (a.rows + a.strip - 1) / a.strip : 0;
}

}  // namespace eqk

extern "C" {

size_t eqlinear_selective_scan_workspace_bytes(const eqlinear_scan_shape* s) {
  eqk::ScanArgs a;
  if (scan_args(s, a, false) || a.B == 0) return 0;
  return scan_carry(a) + scan_sums(a);
}

size_t eqlinear_selective_scan_states_bytes(const eqlinear_scan_shape* s) {
  eqk::ScanArgs a;
  if (scan_args(s, a, false)) return 0;
  return scan_states(a);
}

int eqlinear_selective_scan(const eqlinear_scan_shape* s, const void* x, const void* delta, const float* A, const void* b,
                            const void* c, const float* D, const void* z, const float* delta_bias, const int32_t* lengths,
                            const float* state_in, void* y, float* state_out, float* states, void* workspace,
                            size_t workspace_bytes, void* stream) {
  eqk::ScanArgs a;
  if (int st = scan_args(s, a, false)) return st;
  ScanInputs in;
  if (int st = scan_inputs(s, a, x, delta, A, b, c, D, z, delta_bias, lengths, in)) return st;
  const size_t e = elem_bytes(s->dtype), n = (size_t)a.B * a.L * a.CT * e, hb = (size_t)a.B * a.CT * a.N * 4;
  if (n > 0 && !y) return EQL_ERR_INVALID_ARG;
  if (!aligned(y, e) || !aligned(state_in, 4) || !aligned(state_out, 4) || !aligned(states, 16) || !aligned(workspace, 16))
    return EQL_ERR_ALIGNMENT;
  const size_t need = a.B == 0 ? 0 : scan_carry(a) + scan_sums(a);
  const Range out[4] = {{y, n}, {state_out, hb}, {states, scan_states(a)},
                        {workspace, workspace_bytes < need ? workspace_bytes : need}};
  const Range h0{state_in, hb};
  if (!apart(out, 4, in.r, 9) || overlaps(out[0], h0) || overlaps(out[2], h0) || overlaps(out[3], h0) ||
      (state_in != state_out && overlaps(out[1], h0)))
    return EQL_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  if (a.B == 0) return EQL_OK;
  a.x = x;
  a.delta = delta;
  a.A = A;
  a.b = b;
  a.c = c;
  a.D = D;
  a.z = z;
  a.bias = delta_bias;
  a.lengths = lengths;
  a.h0 = state_in;
  a.y = y;
  a.hT = state_out;
  a.states = states;
  a.carry = (float*)workspace;
  a.sums = (float*)((char*)workspace + scan_carry(a));
  a.mode = scan_mode(a, s->dtype);
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::scan_forward<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::scan_forward<eqk::kF16>(a, st));
  return launched(eqk::scan_forward<eqk::kBF16>(a, st));
}

size_t eqlinear_selective_scan_backward_workspace_bytes(const eqlinear_scan_shape* s) {
  eqk::ScanArgs a;
  if (scan_args(s, a, true)) return 0;
  return scan_carry(a) + scan_sums(a) + scan_part(a) + scan_bcpart(a);
}

int eqlinear_selective_scan_backward(const eqlinear_scan_shape* s, const void* x, const void* delta, const float* A,
                                     const void* b, const void* c, const float* D, const void* z, const float* delta_bias,
                                     const int32_t* lengths, const float* states, const void* dy, const float* d_state_out,
                                     void* dx, void* ddelta, float* dA, void* db, void* dc, float* dD, void* dz,
                                     float* ddelta_bias, float* d_state_in, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  eqk::ScanArgs a;
  if (int st = scan_args(s, a, true)) return st;
  ScanInputs in;
  if (int st = scan_inputs(s, a, x, delta, A, b, c, D, z, delta_bias, lengths, in)) return st;
  const size_t e = elem_bytes(s->dtype), n = (size_t)a.B * a.L * a.CT * e, hb = (size_t)a.B * a.CT * a.N * 4;
  const size_t nb = (size_t)a.B * a.L * a.G * a.N * e;
  if (!dA || (n > 0 && (!dy || !dx || !ddelta || !db || !dc || !states)) || (dz && !z)) return EQL_ERR_INVALID_ARG;
  if (!aligned(dy, e) || !aligned(dx, e) || !aligned(ddelta, e) || !aligned(db, e) || !aligned(dc, e) || !aligned(dz, e) ||
      !aligned(dA, 4) || !aligned(dD, 4) || !aligned(ddelta_bias, 4) || !aligned(d_state_in, 4) || !aligned(d_state_out, 4) ||
      !aligned(states, 16) || !aligned(workspace, 16))
    return EQL_ERR_ALIGNMENT;
  const size_t need = scan_carry(a) + scan_sums(a) + scan_part(a) + scan_bcpart(a);
  const Range out[10] = {{dx, n}, {ddelta, n}, {dz, n}, {db, nb}, {dc, nb}, {dA, (size_t)a.C * a.N * 4},
                         {dD, (size_t)a.C * 4}, {ddelta_bias, (size_t)a.C * 4}, {d_state_in, hb},
                         {workspace, workspace_bytes < need ? workspace_bytes : need}};
  const Range more[3] = {{states, scan_states(a)}, {dy, n}, {d_state_out, hb}};
  if (!apart(out, 10, in.r, 9) || !apart(out, 10, more, 3)) return EQL_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.x = x;
  a.delta = delta;
  a.A = A;
  a.b = b;
  a.c = c;
  a.D = D;
  a.z = z;
  a.bias = delta_bias;
  a.lengths = lengths;
  a.states = const_cast<float*>(states);
  a.dy = dy;
  a.dhT = d_state_out;
  a.dx = dx;
  a.ddelta = ddelta;
  a.dA = dA;
  a.db = db;
  a.dc = dc;
  a.dD = dD;
  a.dz = dz;
  a.dbias = ddelta_bias;
  a.dh0 = d_state_in;
  a.carry = (float*)workspace;
  a.sums = (float*)((char*)workspace + scan_carry(a));
  a.part = (float*)((char*)workspace + scan_carry(a) + scan_sums(a));
  a.bcpart = (float*)((char*)workspace + scan_carry(a) + scan_sums(a) + scan_part(a));
  a.mode = scan_mode(a, s->dtype);
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::scan_backward<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::scan_backward<eqk::kF16>(a, st));
  return launched(eqk::scan_backward<eqk::kBF16>(a, st));
}

}  // extern "C"

// ---- causal convolution ----

namespace {

int conv_args(const eqlinear_conv_shape* s, eqk::ConvArgs& a, bool bwd) {
  if (!s || !valid_dtype(s->dtype) || s->B < 0 || s->L < 0 || s->C < 1 || s->T < 1 || s->W < 1 || s->reserved != 0 ||
      (s->act != EQL_ACT_NONE && s->act != EQL_ACT_SILU))
    return EQL_ERR_INVALID_ARG;
  if (s->T > EQLINEAR_MAX_T || (int64_t)s->C * s->T > kMaxCols || s->W > eqk::kConvMaxW || s->B > kMaxB || s->L > kMaxL ||
      (double)s->B * (double)(s->L + s->W) * s->C * s->T > (double)kMaxElems)
    return EQL_ERR_UNSUPPORTED;
  a = eqk::ConvArgs{};
  a.B = s->B;
  a.L = s->L;
  a.C = s->C;
  a.T = s->T;
  a.W = s->W;
  a.silu = s->act == EQL_ACT_SILU;
  a.xs[0] = s->x_stride[0];
  a.xs[1] = s->x_stride[1];
  eqk::conv_plan(a, s->dtype, kPlanCus, bwd);
  return EQL_OK;
}

size_t conv_part(const eqk::ConvArgs& a) { return align256((size_t)a.B * a.groups * (a.W + 1) * a.CT * sizeof(float)); }

// The inputs of both passes: x, weight, bias, lengths, state.
int conv_inputs(const eqlinear_conv_shape* s, const eqk::ConvArgs& a, const void* x, const void* weight, const void* bias,
                const int32_t* lengths, const void* state_in, Range* r) {
  const size_t e = elem_bytes(s->dtype);
  const int64_t st[3] = {a.xs[0], a.xs[1], 0};
  const int64_t xb = span(a.B, a.L, 1, a.CT, st, e);
  if (xb < 0 || !weight || (xb > 0 && !x)) return EQL_ERR_INVALID_ARG;
  if (!aligned(x, e) || !aligned(weight, e) || !aligned(bias, e) || !aligned(lengths, 4) || !aligned(state_in, e))
    return EQL_ERR_ALIGNMENT;
  r[0] = Range{x, (size_t)xb};
  r[1] = Range{weight, (size_t)a.C * a.W * e};
  r[2] = Range{bias, (size_t)a.C * e};
  r[3] = Range{lengths, (size_t)a.B * 4};
  r[4] = Range{state_in, (size_t)a.B * (a.W - 1) * a.CT * e};
  return EQL_OK;
}

int conv_mode(const eqk::ConvArgs& a, int dtype, bool bwd) {
  const int vec = eqk::conv_vec(dtype, a.W, bwd);
  const size_t e = elem_bytes(dtype);
  const int64_t none[1] = {0};
  const void* dense[7] = {a.h0, a.y, a.hT, a.dy, a.dx, a.dhT, a.dh0};
  bool ok = a.CT % vec == 0 && vectors(a.x, a.xs, 2, e, vec);
  for (const void* p : dense) ok = ok && vectors(p, none, 1, e, vec);
  return ok ? eqk::kWhole : a.CT < vec ? eqk::kTiny : eqk::kLoose;
}

}  // namespace

extern "C" {

int eqlinear_causal_conv(const eqlinear_conv_shape* s, const void* x, const void* weight, const void* bias,
                         const int32_t* lengths, const void* state_in, void* y, void* state_out, void* stream) {
  eqk::ConvArgs a;
  if (int st = conv_args(s, a, false)) return st;
  Range in[5];
  if (int st = conv_inputs(s, a, x, weight, bias, lengths, state_in, in)) return st;
  const size_t e = elem_bytes(s->dtype), n = (size_t)a.B * a.L * a.CT * e;
  if (n > 0 && !y) return EQL_ERR_INVALID_ARG;
  if (!aligned(y, e) || !aligned(state_out, e)) return EQL_ERR_ALIGNMENT;
  const Range out[2] = {{y, n}, {state_out, in[4].bytes}};
  if (!apart(out, 2, in, 4) || overlaps(out[0], in[4]) || (state_in != state_out && overlaps(out[1], in[4])))
    return EQL_ERR_INVALID_ARG;
  if (int st = check_device()) return st;
  if (a.B == 0) return EQL_OK;
  a.x = x;
  a.w = weight;
  a.bias = bias;
  a.lengths = lengths;
  a.h0 = state_in;
  a.y = y;
  a.hT = state_out;
  a.mode = conv_mode(a, s->dtype, false);
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::conv_forward<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::conv_forward<eqk::kF16>(a, st));
  return launched(eqk::conv_forward<eqk::kBF16>(a, st));
}

size_t eqlinear_causal_conv_backward_workspace_bytes(const eqlinear_conv_shape* s) {
  eqk::ConvArgs a;
  if (conv_args(s, a, true)) return 0;
  return conv_part(a);
}

int eqlinear_causal_conv_backward(const eqlinear_conv_shape* s, const void* x, const void* weight, const void* bias,
                                  const int32_t* lengths, const void* state_in, const void* dy, const void* d_state_out,
                                  void* dx, void* dweight, void* dbias, void* d_state_in, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  eqk::ConvArgs a;
  if (int st = conv_args(s, a, true)) return st;
  Range in[7];
  if (int st = conv_inputs(s, a, x, weight, bias, lengths, state_in, in)) return st;
  const size_t e = elem_bytes(s->dtype), n = (size_t)a.B * a.L * a.CT * e, hb = (size_t)a.B * (a.W - 1) * a.CT * e;
  if (!dweight || (n > 0 && (!dy || !dx))) return EQL_ERR_INVALID_ARG;
  if (!aligned(dy, e) || !aligned(d_state_out, e) || !aligned(dx, e) || !aligned(dweight, e) || !aligned(dbias, e) ||
      !aligned(d_state_in, e) || !aligned(workspace, 16))
    return EQL_ERR_ALIGNMENT;
  const size_t need = conv_part(a);
  in[5] = Range{dy, n};
  in[6] = Range{d_state_out, hb};
  const Range out[5] = {{dx, n}, {dweight, (size_t)a.C * a.W * e}, {dbias, (size_t)a.C * e}, {d_state_in, hb},
                        {workspace, workspace_bytes < need ? workspace_bytes : need}};
  if (!apart(out, 5, in, 7)) return EQL_ERR_INVALID_ARG;
  if (need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.x = x;
  a.w = weight;
  a.bias = bias;
  a.lengths = lengths;
  a.h0 = state_in;
  a.dy = dy;
  a.dhT = d_state_out;
  a.dx = dx;
  a.dw = dweight;
  a.db = dbias;
  a.dh0 = d_state_in;
  a.part = (float*)workspace;
  a.mode = conv_mode(a, s->dtype, true);
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::conv_backward<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::conv_backward<eqk::kF16>(a, st));
  return launched(eqk::conv_backward<eqk::kBF16>(a, st));
}

}  // extern "C"

// ---- residual norm ----

namespace {

int res_args(const eqlinear_residual_shape* s, eqk::ResArgs& a) {
  if (!s || !valid_dtype(s->dtype) || s->B < 0 || s->L < 0 || s->C < 1 || s->T < 1 || s->reserved != 0 ||
      (s->kind != EQL_NORM_LAYER && s->kind != EQL_NORM_RMS) || !(s->eps >= 0.0f) || isinf(s->eps))
    return EQL_ERR_INVALID_ARG;
  if (s->T > EQLINEAR_MAX_T || (int64_t)s->C * s->T > eqk::kResMaxRow || s->B > ((int64_t)1 << 31) ||
      s->L > ((int64_t)1 << 36) || (double)s->B * (double)s->L > (double)((int64_t)1 << 36) ||
      (double)s->B * (double)s->L * s->C * s->T > (double)kMaxElems)
    return EQL_ERR_UNSUPPORTED;
  a = eqk::ResArgs{};
  a.B = s->B;
  a.L = s->L;
  a.C = s->C;
  a.T = s->T;
  a.rms = s->kind == EQL_NORM_RMS;
  a.eps = s->eps;
  return EQL_OK;
}

int res_mode(const eqk::ResArgs& a, int dtype) {
  const size_t e = elem_bytes(dtype);
  bool ok = (size_t)a.K * e % 16 == 0;
  const void* rows[8] = {a.x, a.u, a.r, a.h, a.dr, a.dh, a.dx, a.du};
  for (const void* p : rows) ok = ok && aligned(p, 16);
  return ok ? eqk::kWhole : (size_t)a.K * e < 16 ? eqk::kTiny : eqk::kLoose;
}

// rows of column sums: dw and db of a norm after, one or two of a branch
int res_sums(bool weight, bool branch, bool post) { return (weight ? 2 : 0) + (branch ? post ? 2 : 1 : 0); }

size_t res_need(const eqk::ResArgs& a) {
  return align256((size_t)a.seqs * a.strips * a.J * a.K * sizeof(float)) + align256((size_t)a.seqs * a.J * a.C * sizeof(float));
}

}  // namespace

extern "C" {

int eqlinear_residual_norm(const eqlinear_residual_shape* s, const void* x, const void* branch, const void* weight,
                           const void* bias, const void* scale, const void* gate, const void* post_weight,
                           const void* post_bias, void* r, void* h, void* stream) {
  eqk::ResArgs a;
  if (int st = res_args(s, a)) return st;
  const size_t e = elem_bytes(s->dtype), n = (size_t)a.B * a.L * a.C * a.T * e, p = (size_t)a.C * e;
  if (!branch && (scale || gate || post_weight || r) && n > 0) return EQL_ERR_INVALID_ARG;
  if ((bias && !weight) || (post_bias && !post_weight) || (n > 0 && (!x || (branch && !r) || (weight && !h) || (!branch && !weight))))
    return EQL_ERR_INVALID_ARG;
  const void* every[10] = {x, branch, weight, bias, scale, gate, post_weight, post_bias, r, h};
  for (const void* q : every)
    if (!aligned(q, e)) return EQL_ERR_ALIGNMENT;
  const Range out[2] = {{r, n}, {h, weight ? n : 0}};
  const Range in[8] = {{x, n}, {branch, n}, {weight, p}, {bias, p}, {scale, p}, {gate, (size_t)a.B * p}, {post_weight, p}, {post_bias, p}};
  if (!apart(out, 2, in, 8)) return EQL_ERR_INVALID_ARG;
  if (int st = check_device()) return st;
  if (n == 0) return EQL_OK;
  a.x = x;
  a.u = branch;
  a.w = weight;
  a.b = bias;
  a.scale = scale;
  a.gate = gate;
  a.pw = post_weight;
  a.pb = post_bias;
  a.r = r;
  a.h = h;
  eqk::res_plan(a, s->dtype, kPlanCus, false);
  a.mode = res_mode(a, s->dtype);
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::res_forward<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::res_forward<eqk::kF16>(a, st));
  return launched(eqk::res_forward<eqk::kBF16>(a, st));
}

// The most that any choice of parameters needs: a call with fewer uses less of it.
size_t eqlinear_residual_norm_backward_workspace_bytes(const eqlinear_residual_shape* s) {
  eqk::ResArgs a;
  if (res_args(s, a) || a.B == 0) return 0;
  a.J = res_sums(true, true, true);
  eqk::res_plan(a, s->dtype, kPlanCus, true);
  const size_t one = res_need(a);
  a.gate = s;  // (any address: sequences on their own)
  eqk::res_plan(a, s->dtype, kPlanCus, true);
  const size_t each = res_need(a);
  return one > each ? one : each;
}

int eqlinear_residual_norm_backward(const eqlinear_residual_shape* s, const void* x, const void* branch, const void* weight,
                                    const void* scale, const void* gate, const void* post_weight, const void* post_bias,
                                    const void* dr, const void* dh, void* dx, void* dbranch, void* dweight, void* dbias,
                                    void* dscale, void* dgate, void* dpost_weight, void* dpost_bias, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  eqk::ResArgs a;
  if (int st = res_args(s, a)) return st;
  const size_t e = elem_bytes(s->dtype), n = (size_t)a.B * a.L * a.C * a.T * e, p = (size_t)a.C * e;
  if (!branch && (scale || gate || post_weight || dbranch) && n > 0) return EQL_ERR_INVALID_ARG;
  if ((post_bias && !post_weight) || (dh && !weight) || ((dweight || dbias) && !weight) || (dscale && !scale) ||
      (dgate && !gate) || ((dpost_weight || dpost_bias) && !post_weight) || (n > 0 && !x))
    return EQL_ERR_INVALID_ARG;
  const void* every[17] = {x, branch, weight, scale, gate, post_weight, post_bias, dr, dh, dx, dbranch, dweight, dbias,
                           dscale, dgate, dpost_weight, dpost_bias};
  for (const void* q : every)
    if (!aligned(q, e)) return EQL_ERR_ALIGNMENT;
  if (!aligned(workspace, 16)) return EQL_ERR_ALIGNMENT;
  a.x = x;
  a.u = branch;
  a.w = weight;
  a.scale = scale;
  a.gate = gate;
  a.pw = post_weight;
  a.pb = post_bias;
  a.dr = dr;
  a.dh = dh;
  a.dx = dx;
  a.du = dbranch;
  a.dw = dweight;
  a.db = dbias;
  a.dscale = dscale;
  a.dgate = dgate;
  a.dpw = dpost_weight;
  a.dpb = dpost_bias;
  a.J = res_sums(weight, branch, post_weight);
  eqk::res_plan(a, s->dtype, kPlanCus, true);
  const size_t need = res_need(a);
  const Range out[9] = {{dx, n}, {dbranch, n}, {dweight, p}, {dbias, p}, {dscale, p}, {dgate, (size_t)a.B * p},
                        {dpost_weight, p}, {dpost_bias, p}, {workspace, workspace_bytes < need ? workspace_bytes : need}};
  const Range in[9] = {{x, n}, {branch, n}, {weight, p}, {scale, p}, {gate, (size_t)a.B * p}, {post_weight, p}, {post_bias, p},
                       {dr, n}, {dh, n}};
  if (!apart(out, 9, in, 9)) return EQL_ERR_INVALID_ARG;
  if (n > 0 && need > 0 && (!workspace || workspace_bytes < need)) return EQL_ERR_WORKSPACE;
  if (int st = check_device()) return st;
  a.part = (float*)workspace;
  a.sums = (float*)((char*)workspace + align256((size_t)a.seqs * a.strips * a.J * a.K * sizeof(float)));
  a.mode = res_mode(a, s->dtype);
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == EQL_F32) return launched(eqk::res_backward<eqk::kF32>(a, st));
  if (s->dtype == EQL_F16) return launched(eqk::res_backward<eqk::kF16>(a, st));
  return launched(eqk::res_backward<eqk::kBF16>(a, st));
}

}  // extern "C"
