// eql_scan.hip -- selective scan (eql_scan.h): instantiations, plans and launches of
// one element type (EQK_DT).
#include "eql_scan.h"
#include "eql_launch.h"

namespace eqk {
namespace {

constexpr int DT = EQK_DT;

// f(slice of the sequences that one launch takes, its number of sequences); `waves`: of a sequence
template <typename F>
hipError_t sequences(const ScanArgs& a, int64_t waves, F&& f) {
  ScanArgs s = a;
  const int64_t most = ((int64_t)1 << 30) / (64 * waves);  // (below 2^32 threads, and numbers of 31 bits)
  if (most < 1) return hipErrorInvalidValue;
  for (s.first = 0; s.first < a.B; s.first += most) {
    f(s, a.B - s.first < most ? a.B - s.first : most);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// f(the call from `first` on, workgroups of 256) for `n` elements, or workgroups where per is 1
template <typename F>
hipError_t elements(const ScanArgs& a, int64_t n, int per, F&& f) {
  ScanArgs s = a;
  const int64_t most = launch_blocks(256) * per;
  for (s.first = 0; s.first < n; s.first += most) {
    f(s, dim3((unsigned)(((n - s.first < most ? n - s.first : most) + per - 1) / per)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
dim3 wave_blocks(ScanArgs& s, int64_t seqs, int blocks) {
  s.tasks = (unsigned)(seqs * s.K * s.G * blocks);
  return dim3((s.tasks + kScanWaves - 1) / kScanWaves);
}

template <int NL, int MODE>
hipError_t fwd(const ScanArgs& a, hipStream_t stream) {
  const int64_t waves = (int64_t)a.K * a.G * a.bblk;
  if (a.K > 1) {
    hipError_t e = sequences(a, waves, [&](ScanArgs s, int64_t n) {
      const dim3 g = wave_blocks(s, n, s.bblk);
      hipLaunchKernelGGL((eql_scan_fwd_kernel<DT, NL, MODE, true>), g, dim3(64 * kScanWaves), 0, stream, s);
    });
    if (e != hipSuccess) return e;
    e = sequences(a, a.cols * NL / 16, [&](const ScanArgs& s, int64_t n) {
      hipLaunchKernelGGL(eql_scan_carry_kernel<false>, dim3((unsigned)(n * (a.cols * NL / 16))), dim3(64), 0, stream, s, 4 * NL);
    });
    if (e != hipSuccess) return e;
  }
  return sequences(a, waves, [&](ScanArgs s, int64_t n) {
    const dim3 g = wave_blocks(s, n, s.bblk);
    hipLaunchKernelGGL((eql_scan_fwd_kernel<DT, NL, MODE, false>), g, dim3(64 * kScanWaves), 0, stream, s);
  });
}

template <int NL, int MODE>
hipError_t bwd(const ScanArgs& a, hipStream_t stream) {
  hipError_t e;
  if (a.K > 1) {
    e = sequences(a, (int64_t)a.K * a.G * a.bblk, [&](ScanArgs s, int64_t n) {
      const dim3 g = wave_blocks(s, n, s.bblk);
      hipLaunchKernelGGL((eql_scan_back_kernel<DT, NL, MODE>), g, dim3(64 * kScanWaves), 0, stream, s);
    });
    if (e != hipSuccess) return e;
    e = sequences(a, a.cols * NL / 16, [&](const ScanArgs& s, int64_t n) {
      hipLaunchKernelGGL(eql_scan_carry_kernel<true>, dim3((unsigned)(n * (a.cols * NL / 16))), dim3(64), 0, stream, s, 4 * NL);
    });
    if (e != hipSuccess) return e;
  }
  auto k = eql_scan_bwd_kernel<DT, NL, MODE>;
  const int waves = a.waves, lds = scan_bwd_bytes<NL>(waves);
  if (lds > 65536) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  const int64_t per = (int64_t)a.K * a.G * a.P;
  e = sequences(a, per * waves, [&](const ScanArgs& s, int64_t n) {
    hipLaunchKernelGGL(k, dim3((unsigned)(n * per)), dim3(64 * waves), lds, stream, s, waves);
  });
  if (e != hipSuccess) return e;
  if (a.P > 1) {
    e = elements(a, a.B * a.L * a.G * 8 * NL, 256, [&](const ScanArgs& s, dim3 n) {
      hipLaunchKernelGGL(eql_scan_bc_kernel<DT>, n, dim3(256), 0, stream, s, 4 * NL);
    });
    if (e != hipSuccess) return e;
  }
  return elements(a, (int64_t)a.C * (a.N + 2), 1, [&](const ScanArgs& s, dim3 n) {
    hipLaunchKernelGGL(eql_scan_params_kernel<>, n, dim3(256), 0, stream, s, scan_cols(NL));
  });
}

template <int NL>
hipError_t few(const ScanArgs& a, hipStream_t stream) {
  return sequences(a, (int64_t)a.G * a.nblk, [&](ScanArgs s, int64_t n) {
    const dim3 g = wave_blocks(s, n, s.nblk);
    hipLaunchKernelGGL((eql_scan_few_kernel<DT, NL>), g, dim3(64 * kScanWaves), 0, stream, s);
  });
}

template <int NL>
hipError_t pass(const ScanArgs& a, bool back, hipStream_t stream) {
  if (!back && a.L <= scan_few(NL) && !a.states) return few<NL>(a, stream);
  if (a.mode == kWhole) return back ? bwd<NL, kWhole>(a, stream) : fwd<NL, kWhole>(a, stream);
  if (a.mode == kLoose) return back ? bwd<NL, kLoose>(a, stream) : fwd<NL, kLoose>(a, stream);
  return back ? bwd<NL, kTiny>(a, stream) : fwd<NL, kTiny>(a, stream);
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
