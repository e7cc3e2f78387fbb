// eql_recurrent.hip -- plans of the recurrent operators; instantiations and launches of the causal
// convolution (eql_conv.h) and the residual norm (eql_resnorm.h) of one element type (EQK_DT).
#include "eql_conv.h"
#include "eql_launch.h"
#include "eql_resnorm.h"

namespace eqk {
namespace {

constexpr int DT = EQK_DT;

// f(slice of the call that one launch takes, its workgroups)
template <typename A, typename F>
hipError_t launches(const A& a, int64_t blocks, int threads, F&& f) {
  A s = a;
  const int64_t most = launch_blocks(threads);
  for (s.first = 0; s.first < blocks; s.first += most) {
    f(s, dim3((unsigned)(blocks - s.first < most ? blocks - s.first : most)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int W, bool BACK, bool WHOLE>
hipError_t conv_w(const ConvArgs& a, hipStream_t stream) {
  constexpr int VEC = conv_vec(DT, W, BACK);
  const int64_t threads = a.B * a.strips * ((a.CT + VEC - 1) / VEC);
  const hipError_t e = launches(a, (threads + 255) / 256, 256, [&](const ConvArgs& s, dim3 n) {
    if constexpr (BACK) hipLaunchKernelGGL((eql_conv_bwd_kernel<DT, W, VEC, WHOLE>), n, dim3(256), 0, stream, s);
    else hipLaunchKernelGGL((eql_conv_fwd_kernel<DT, W, VEC, WHOLE>), n, dim3(256), 0, stream, s);
  });
  if (e != hipSuccess || !BACK) return e;
  return launches(a, (int64_t)a.C * (W + 1), 256, [&](const ConvArgs& s, dim3 n) {
    hipLaunchKernelGGL(eql_conv_params_kernel<DT>, n, dim3(256), 0, stream, s);
  });
}
template <bool BACK, int W = 1>
hipError_t conv(const ConvArgs& a, hipStream_t stream) {
  if constexpr (W > kConvMaxW) {
    return hipErrorInvalidValue;
  } else {
    if (a.W != W) return conv<BACK, W + 1>(a, stream);
    return a.vec > 1 ? conv_w<W, BACK, true>(a, stream) : conv_w<W, BACK, false>(a, stream);
  }
}

template <int LANES, int EPT, bool WHOLE>
hipError_t res_row(const ResArgs& a, bool back, hipStream_t stream) {
  constexpr int threads = ResRow<DT, LANES, EPT, WHOLE>::THREADS;
  return launches(a, a.seqs * a.strips, threads, [&](const ResArgs& s, dim3 n) {
    if (back) hipLaunchKernelGGL((eql_res_bwd_kernel<DT, LANES, EPT, WHOLE>), n, dim3(threads), 0, stream, s);
    else hipLaunchKernelGGL((eql_res_fwd_kernel<DT, LANES, EPT, WHOLE>), n, dim3(threads), 0, stream, s);
  });
}
template <bool WHOLE>
hipError_t res_lanes(const ResArgs& a, bool back, hipStream_t stream) {
  if (a.lanes == 16) return res_row<16, 8, WHOLE>(a, back, stream);
  if (a.lanes == 64) return a.ept == 8 ? res_row<64, 8, WHOLE>(a, back, stream) : res_row<64, 16, WHOLE>(a, back, stream);
  if (a.lanes == 256) return a.ept == 8 ? res_row<256, 8, WHOLE>(a, back, stream) : res_row<256, 16, WHOLE>(a, back, stream);
  return res_row<512, 16, WHOLE>(a, back, stream);
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
  return a.whole ? res_lanes<true>(a, false, stream) : res_lanes<false>(a, false, stream);
}
template <>
hipError_t res_backward<DT>(const ResArgs& a, hipStream_t stream) {
  const hipError_t e = a.seqs * a.rows == 0 ? hipSuccess : a.whole ? res_lanes<true>(a, true, stream) : res_lanes<false>(a, true, stream);
  if (e != hipSuccess || a.J == 0) return e;
  const hipError_t f = launches(a, a.seqs * a.J * a.C, 256, [&](const ResArgs& s, dim3 n) {
    hipLaunchKernelGGL(eql_res_strips_kernel<>, n, dim3(256), 0, stream, s);
  });
  if (f != hipSuccess) return f;
  return launches(a, (a.C + 3) / 4, 256, [&](const ResArgs& s, dim3 n) {
    hipLaunchKernelGGL(eql_res_params_kernel<DT>, n, dim3(256), 0, stream, s);
  });
}

}  // namespace eqk
