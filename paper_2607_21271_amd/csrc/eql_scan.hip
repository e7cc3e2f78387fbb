// eql_scan.hip -- selective scan (eql_scan.h): instantiations, plans and launches of
// one element type (EQK_DT).
#include "eql_scan.h"
#include "eql_launch.h"

namespace eqk {
namespace {

constexpr int DT = EQK_DT;

// f(slice of the call that one launch takes, its workgroups)
template <typename F>
hipError_t launches(const ScanArgs& a, int64_t blocks, int threads, F&& f) {
  ScanArgs s = a;
  const int64_t most = launch_blocks(threads);
  for (s.first = 0; s.first < blocks; s.first += most) {
    f(s, dim3((unsigned)(blocks - s.first < most ? blocks - s.first : most)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int NL, bool WHOLE>
hipError_t fwd(const ScanArgs& a, hipStream_t stream) {
  const int64_t blocks = (a.B * a.K * a.G * a.nblk + kScanWaves - 1) / kScanWaves;
  if (a.K > 1) {
    hipError_t e = launches(a, blocks, 256, [&](const ScanArgs& s, dim3 n) {
      hipLaunchKernelGGL((eql_scan_fwd_kernel<DT, NL, WHOLE, true>), n, dim3(256), 0, stream, s);
    });
    if (e != hipSuccess) return e;
    e = launches(a, (a.B * a.cols * 4 * NL + 255) / 256, 256, [&](const ScanArgs& s, dim3 n) {
      hipLaunchKernelGGL(eql_scan_carry_kernel<false>, n, dim3(256), 0, stream, s, 4 * NL);
    });
    if (e != hipSuccess) return e;
  }
  return launches(a, blocks, 256, [&](const ScanArgs& s, dim3 n) {
    hipLaunchKernelGGL((eql_scan_fwd_kernel<DT, NL, WHOLE, false>), n, dim3(256), 0, stream, s);
  });
}

template <int NL, bool WHOLE>
hipError_t bwd(const ScanArgs& a, hipStream_t stream) {
  hipError_t e;
  if (a.K > 1) {
    e = launches(a, (a.B * a.K * a.G * a.nblk + kScanWaves - 1) / kScanWaves, 256, [&](const ScanArgs& s, dim3 n) {
      hipLaunchKernelGGL((eql_scan_back_kernel<DT, NL, WHOLE>), n, dim3(256), 0, stream, s);
    });
    if (e != hipSuccess) return e;
    e = launches(a, (a.B * a.cols * 4 * NL + 255) / 256, 256, [&](const ScanArgs& s, dim3 n) {
      hipLaunchKernelGGL(eql_scan_carry_kernel<true>, n, dim3(256), 0, stream, s, 4 * NL);
    });
    if (e != hipSuccess) return e;
  }
  constexpr int SUB = scan_tile(NL) < 8 ? scan_tile(NL) : 8;
  auto k = eql_scan_bwd_kernel<DT, NL, WHOLE, SUB>;
  const int waves = a.nblk < kScanWaves ? a.nblk : kScanWaves, lds = scan_bwd_bytes<NL>(waves);
  if (lds > 65536) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  e = launches(a, a.B * a.K * a.G * a.P, 64 * waves, [&](const ScanArgs& s, dim3 n) {
    hipLaunchKernelGGL(k, n, dim3(64 * waves), lds, stream, s, waves);
  });
  if (e != hipSuccess) return e;
  if (a.P > 1) {
    e = launches(a, (a.B * a.L * a.G * 8 * NL + 255) / 256, 256, [&](const ScanArgs& s, dim3 n) {
      hipLaunchKernelGGL(eql_scan_bc_kernel<DT>, n, dim3(256), 0, stream, s, 4 * NL);
    });
    if (e != hipSuccess) return e;
  }
  return launches(a, (int64_t)a.C * (a.N + 2), 256, [&](const ScanArgs& s, dim3 n) {
    hipLaunchKernelGGL(eql_scan_params_kernel<>, n, dim3(256), 0, stream, s, scan_cols(NL));
  });
}

template <int NL>
hipError_t pass(const ScanArgs& a, bool back, hipStream_t stream) {
  if (a.whole) return back ? bwd<NL, true>(a, stream) : fwd<NL, true>(a, stream);
  return back ? bwd<NL, false>(a, stream) : fwd<NL, false>(a, stream);
}

hipError_t run(const ScanArgs& a, bool back, hipStream_t stream) {
  switch (scan_lanes(a.N)) {
    case 1: return pass<1>(a, back, stream);
    case 2: return pass<2>(a, back, stream);
    case 4: return pass<4>(a, back, stream);
    case 8: return pass<8>(a, back, stream);
    default: return pass<16>(a, back, stream);
  }
}

}  // namespace

template <>
hipError_t scan_forward<DT>(const ScanArgs& a, hipStream_t stream) {
  return run(a, false, stream);
}
template <>
hipError_t scan_backward<DT>(const ScanArgs& a, hipStream_t stream) {
  return run(a, true, stream);
}

}  // namespace eqk
