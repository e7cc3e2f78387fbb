// eql_recurrent.h -- arguments, plans and launches of the scan, causal convolution and
// residual-norm kernels, shared by host and device code.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eql_config.h"

namespace eqk {

// The channel of column ct <= 65536 in rows of T group elements, T <= 16: ct m / 2^21 with m = ceil(2^21 / T), which is
// off by less than the 1 / T that it may be.
constexpr unsigned channel_factor(int T) { return (unsigned)(((1 << 21) + T - 1) / T); }
__device__ __forceinline__ int channel_of(int ct, unsigned m) { return (int)__umulhi((unsigned)ct << 11, m); }

// How rows are read and written (eql_vectors.h, ScanTile).
constexpr int kWhole = 0, kLoose = 1, kTiny = 2;

// ---- selective scan ----
// A wave takes `scan_cols(NL, Q)` neighbouring columns (channel, group element) of one group: NL lanes share Q columns and
// hold four states of each.  Q is scan_columns(NL) in the kernels of tiles, forward and gradients, four in the one of few
// tokens.  A group's columns are padded to whole scan_cols(NL) in what is kept for them (states, carry, sums).
constexpr int kScanMaxN = 64;
constexpr int scan_lanes(int N) { return N <= 4 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }
constexpr int scan_cols(int NL, int Q = 4) { return 64 * Q / NL; }
// columns of a lane in the kernels of tiles
constexpr int scan_columns(int NL) { return NL == 16 ? 4 : 2; }
// tokens of a tile, and of a run, whose first state training keeps
constexpr int scan_tile(int NL) { return NL == 1 ? 4 : NL == 2 ? 8 : 16; }
constexpr int scan_run(int NL) { return NL == 1 ? 4 : 8; }
constexpr int scan_ept(int NL, int Q = 4) { return scan_tile(NL) * scan_cols(NL, Q) / 64; }  // elements of a lane
constexpr int scan_vec(int dt, int NL, int Q = 4) {
  return (dt == kF32 ? 4 : 8) < scan_ept(NL, Q) ? (dt == kF32 ? 4 : 8) : scan_ept(NL, Q);
}
constexpr int kScanWaves = 4;  // of a workgroup

struct ScanArgs {
  const void *x, *delta, *z, *b, *c, *dy;
  const float *A, *D, *bias, *h0, *dhT;
  void *y, *dx, *ddelta, *dz, *db, *dc;
  float *hT, *dh0, *dA, *dD, *dbias;
  const int* lengths;
  float* states;  // [B, runs, cols, NP]: the state before each run
  float* carry;   // [B, K, cols, NP]: the state before each chunk (backward: the gradient behind it)
  float* sums;    // [B, K, cols]: the chunk's sum of d
  float* part;    // [B * K, N + 2, cols]: sums of dA, dD, ddelta_bias
  float* bcpart;  // [B, L, groups, P, 2, NP]: db and dc of each workgroup's columns
  int64_t xs[2], ds[2], zs[2], bs[3], cs[3];
  int64_t B, L;
  int64_t first;         // what a launch starts with: a sequence (an element or workgroup of the small kernels)
  unsigned tasks;        // waves of a launch
  unsigned mT;           // channel_factor(T)
  int64_t chunk, tiles, runs;  // tokens of a chunk (whole tiles), tiles and runs of a sequence
  int C, T, N, G, CT, CTg, nblk, cols, K, softplus;
  int bblk;      // blocks of a group's columns in the kernels of tiles (nblk: of few tokens)
  int waves, P;  // of a workgroup of the gradients, and those side by side for a group's columns
  int mode;  // how rows are read and written (ScanTile)
};

// Fills CT .. P, chunk and tiles for the forward or the backward pass.
void scan_plan(ScanArgs& a, int cus, bool bwd);
template <int DT>
hipError_t scan_forward(const ScanArgs& a, hipStream_t stream);
template <int DT>
hipError_t scan_backward(const ScanArgs& a, hipStream_t stream);
template <> hipError_t scan_forward<kF32>(const ScanArgs&, hipStream_t);
template <> hipError_t scan_forward<kF16>(const ScanArgs&, hipStream_t);
template <> hipError_t scan_forward<kBF16>(const ScanArgs&, hipStream_t);
template <> hipError_t scan_backward<kF32>(const ScanArgs&, hipStream_t);
template <> hipError_t scan_backward<kF16>(const ScanArgs&, hipStream_t);
template <> hipError_t scan_backward<kBF16>(const ScanArgs&, hipStream_t);

// ---- causal convolution ----
constexpr int kConvMaxW = 8;

struct ConvArgs {
  const void *x, *w, *bias, *h0, *dy, *dhT;
  void *y, *hT, *dx, *dw, *db, *dh0;
  const int* lengths;
  float* part;  // [B * groups, W + 1, CT / GR]
  int64_t xs[2];
  int64_t B, L, strips, groups;
  int64_t seq;           // what a launch starts with: a sequence, and a workgroup from it on
  unsigned first;
  unsigned mT;           // channel_factor(T)
  int C, T, W, CT, silu, mode;
  int rows;              // tokens of a strip
  int width, cblocks;    // vectors of columns of a workgroup, workgroups side by side
  int turns;             // strips of a workgroup; `groups` of them are a sequence's
};

constexpr int conv_vec(int dt, int W, bool bwd) { return dt == kF32 ? 4 : bwd && W > 4 ? 4 : 8; }
void conv_plan(ConvArgs& a, int dt, int cus, bool bwd);
template <int DT>
hipError_t conv_forward(const ConvArgs& a, hipStream_t stream);
template <int DT>
hipError_t conv_backward(const ConvArgs& a, hipStream_t stream);
template <> hipError_t conv_forward<kF32>(const ConvArgs&, hipStream_t);
template <> hipError_t conv_forward<kF16>(const ConvArgs&, hipStream_t);
template <> hipError_t conv_forward<kBF16>(const ConvArgs&, hipStream_t);
template <> hipError_t conv_backward<kF32>(const ConvArgs&, hipStream_t);
template <> hipError_t conv_backward<kF16>(const ConvArgs&, hipStream_t);
template <> hipError_t conv_backward<kBF16>(const ConvArgs&, hipStream_t);

// ---- residual norm ----
constexpr int kResMaxRow = 8192;

struct ResArgs {
  const void *x, *u, *w, *b, *scale, *gate, *pw, *pb, *dr, *dh;
  void *r, *h, *dx, *du, *dw, *db, *dscale, *dgate, *dpw, *dpb;
  float* part;  // [seqs, strips, J, K / GR]: column sums of each workgroup
  float* sums;  // [seqs, J, C]
  int64_t B, L;
  int64_t seqs, rows;    // sequences with a gate of their own (else one), tokens of each
  int64_t strips, strip; // workgroups of a sequence and tokens of each
  int64_t seq;     // what a launch starts with: a sequence, and a workgroup from it on
  unsigned first;
  unsigned mT;           // channel_factor(T)
  int C, T, K, rms, J;
  float eps;
  int mode, lanes, ept;  // threads of a row and elements of each
};

void res_plan(ResArgs& a, int dt, int cus, bool bwd);
template <int DT>
hipError_t res_forward(const ResArgs& a, hipStream_t stream);
template <int DT>
hipError_t res_backward(const ResArgs& a, hipStream_t stream);
template <> hipError_t res_forward<kF32>(const ResArgs&, hipStream_t);
template <> hipError_t res_forward<kF16>(const ResArgs&, hipStream_t);
template <> hipError_t res_forward<kBF16>(const ResArgs&, hipStream_t);
template <> hipError_t res_backward<kF32>(const ResArgs&, hipStream_t);
template <> hipError_t res_backward<kF16>(const ResArgs&, hipStream_t);
template <> hipError_t res_backward<kBF16>(const ResArgs&, hipStream_t);

}  // namespace eqk
