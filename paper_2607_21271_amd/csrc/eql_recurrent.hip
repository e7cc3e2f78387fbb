// eql_recurrent.hip -- plans of the recurrent operators; instantiations and launches of the causal
// convolution (eql_conv.h) and the residual norm (eql_resnorm.h) of one element type (EQK_DT).
#include "eql_conv.h"
#include "eql_launch.h"
#include "eql_resnorm.h"
#include "eql_slices.h"

namespace eqk {
namespace {

constexpr int DT = EQK_DT;

// f(slice of the call that one launch takes, its workgroups) for `per` workgroups a sequence: fewer than 2^32
// threads a launch.
template <typename A, typename F>
hipError_t launches(const A& a, int64_t seqs, int64_t per, int threads, F&& f) {
  if (per < 1 || per > kSliceReach) return hipErrorInvalidValue;
  A s = a;
  hipError_t e = hipSuccess;
  slices(seqs, per, launch_blocks(threads), kSliceReach, [&](int64_t seq, unsigned first, unsigned blocks) {
    s.seq = seq;
    s.first = first;
    f(s, dim3(blocks));
    e = hipGetLastError();
    return e == hipSuccess;
  });
  return e;
}

template <int W, bool BACK, int GR, int MODE>
hipError_t conv_gr(const ConvArgs& a, hipStream_t stream) {
  constexpr int VEC = conv_vec(DT, W, BACK);
  if constexpr (GR > VEC) {
    return hipErrorInvalidValue;
  } else {
    const hipError_t e = launches(a, a.B, a.groups * a.cblocks, 256, [&](const ConvArgs& s, dim3 n) {
      if constexpr (BACK) hipLaunchKernelGGL((eql_conv_bwd_kernel<DT, W, VEC, GR, MODE>), n, dim3(256), 0, stream, s);
      else hipLaunchKernelGGL((eql_conv_fwd_kernel<DT, W, VEC, GR, MODE>), n, dim3(256), 0, stream, s);
    });
    if (e != hipSuccess || !BACK) return e;
    hipLaunchKernelGGL(eql_conv_params_kernel<DT>, dim3((unsigned)((W + 1) * colsum_blocks(a.C, a.T / GR))), dim3(kColsumThreads), 0, stream, a, GR);
    return hipGetLastError();
  }
}
template <int W, bool BACK>
hipError_t conv_w(const ConvArgs& a, hipStream_t stream) {
  constexpr int VEC = conv_vec(DT, W, BACK);
  if (a.mode == kTiny) return conv_gr<W, BACK, 1, kTiny>(a, stream);
  if (a.mode == kLoose) return conv_gr<W, BACK, 1, kLoose>(a, stream);
  if (a.T % VEC == 0) return conv_gr<W, BACK, VEC, kWhole>(a, stream);
  if constexpr (VEC == 8)
    if (a.T % 4 == 0) return conv_gr<W, BACK, 4, kWhole>(a, stream);
  return conv_gr<W, BACK, 1, kWhole>(a, stream);
}
template <bool BACK, int W = 1>
hipError_t conv(const ConvArgs& a, hipStream_t stream) {
  if constexpr (W > kConvMaxW) {
    return hipErrorInvalidValue;
  } else {
    return a.W == W ? conv_w<W, BACK>(a, stream) : conv<BACK, W + 1>(a, stream);
  }
}

template <int LANES, int EPT, int MODE, int GR>
hipError_t res_row(const ResArgs& a, bool back, hipStream_t stream) {
  constexpr int threads = ResRow<DT, LANES, EPT, MODE, GR>::THREADS;
  return launches(a, a.seqs, a.strips, threads, [&](const ResArgs& s, dim3 n) {
    if (back) hipLaunchKernelGGL((eql_res_bwd_kernel<DT, LANES, EPT, MODE, GR>), n, dim3(threads), 0, stream, s);
    else hipLaunchKernelGGL((eql_res_fwd_kernel<DT, LANES, EPT, MODE, GR>), n, dim3(threads), 0, stream, s);
  });
}
template <int MODE, int GR>
hipError_t res_lanes(const ResArgs& a, bool back, hipStream_t stream) {
  if (a.lanes == 8) return res_row<8, 8, MODE, GR>(a, back, stream);
  if (a.lanes == 32) return res_row<32, 8, MODE, GR>(a, back, stream);
  if (a.lanes == 4) return res_row<4, 8, MODE, GR>(a, back, stream);
  if (a.lanes == 16) return res_row<16, 8, MODE, GR>(a, back, stream);
  if (a.lanes == 64) return a.ept == 8 ? res_row<64, 8, MODE, GR>(a, back, stream) : res_row<64, 16, MODE, GR>(a, back, stream);
  if (a.lanes == 256) return a.ept == 8 ? res_row<256, 8, MODE, GR>(a, back, stream) : res_row<256, 16, MODE, GR>(a, back, stream);
  return res_row<1024, 8, MODE, GR>(a, back, stream);
}
// columns that share a channel, of a vector
int res_gr(const ResArgs& a) {
  if (a.mode != kWhole) return 1;
  if (DT != kF32 && a.T % 8 == 0) return 8;
  return a.T % 4 == 0 ? 4 : 1;
}
hipError_t res(const ResArgs& a, bool back, hipStream_t stream) {
  const int gr = res_gr(a);
  if constexpr (DT != kF32)
    if (gr == 8) return res_lanes<kWhole, 8>(a, back, stream);
  if (gr == 4) return res_lanes<kWhole, 4>(a, back, stream);
  if (a.mode == kTiny) return res_row<4, 8, kTiny, 1>(a, back, stream);
  return a.mode == kWhole ? res_lanes<kWhole, 1>(a, back, stream) : res_lanes<kLoose, 1>(a, back, stream);
}

}  // namespace

template <>
hipError_t conv_forward<DT>(const ConvArgs& a, hipStream_t stream) {
  return conv<false>(a, stream);
}
template <>
hipError_t conv_backward<DT>(const ConvArgs& a, hipStream_t stream) {
  return conv<true>(a, stream);
}
template <>
hipError_t res_forward<DT>(const ResArgs& a, hipStream_t stream) {
  return res(a, false, stream);
}
template <>
hipError_t res_backward<DT>(const ResArgs& a, hipStream_t stream) {
  if (a.seqs > 0 && a.rows > 0) {  // (else the parameters' gradients are 0)
    hipError_t e = res(a, true, stream);
    if (e != hipSuccess || a.J == 0) return e;
    const int gr = res_gr(a), blocks = colsum_blocks(a.C, a.T / gr);
    e = launches(a, a.seqs, (int64_t)a.J * blocks, kColsumThreads, [&](const ResArgs& s, dim3 n) {
      hipLaunchKernelGGL(eql_res_strips_kernel<>, n, dim3(kColsumThreads), 0, stream, s, gr, blocks);
    });
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(eql_res_params_kernel<DT>, dim3((unsigned)((a.C + kResParamChannels - 1) / kResParamChannels)),
                     dim3(kResParamThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace eqk
