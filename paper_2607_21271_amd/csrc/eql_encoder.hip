// eql_encoder.hip -- instantiations and launches of the rotary (eql_rotary.h) and
// group-norm (eql_gnact.h) kernels.
#include "eql_encoder.h"
#include "eql_launch.h"

namespace eqk {
namespace {

template <int DT, int VEC>
hipError_t rotary_v(const RotaryArgs& a, hipStream_t stream) {
  auto k = eql_rotary_kernel<DT, VEC, false>;
  if constexpr (VEC > 1)
    if (a.interleaved && a.T == 1) k = eql_rotary_kernel<DT, VEC, true>;
  RotaryArgs s = a;
  for (s.first = 0; s.first < a.tokens; s.first += launch_blocks(256) * a.TB) {
    int64_t blocks = (a.tokens - s.first + a.TB - 1) / a.TB;
    if (blocks > launch_blocks(256)) blocks = launch_blocks(256);
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(256), 0, stream, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int DT>
hipError_t rotary_dt(const RotaryArgs& a, int vec, hipStream_t stream) {
  if constexpr (DT != kF32)
    if (vec == 8) return rotary_v<DT, 8>(a, stream);
  if (vec == 4) return rotary_v<DT, 4>(a, stream);
  if (vec == 2) return rotary_v<DT, 2>(a, stream);
  return rotary_v<DT, 1>(a, stream);
}

// The sequences b0 .. b0 + n of a call.  The parts are those of either pass (bwd), the sums stay
// the call's: dw and db add them over all sequences.
template <int DT>
GnArgs gn_slice(const GnArgs& a, int64_t b0, int64_t n, bool bwd) {
  const int64_t at = b0 * a.S * a.K * (int64_t)sizeof(typename Elem<DT>::T);
  GnArgs s = a;
  s.B = n;
  s.x = (const char*)a.x + at;
  if (a.y) s.y = (char*)a.y + at;
  if (a.dy) s.dy = (const char*)a.dy + at;
  if (a.dx) s.dx = (char*)a.dx + at;
  if (a.stats) s.stats = a.stats + b0 * a.G * 2;
  if (a.part) s.part = a.part + (bwd ? b0 * a.chunks * a.C : b0 * a.chunks * a.cblocks * a.G) * 2;
  if (a.sums) s.sums = a.sums + b0 * a.C * 2;
  return s;
}
// f(slice) for slices of at most `most` sequences, until one fails
template <int DT, typename F>
hipError_t gn_slices(const GnArgs& a, int64_t most, bool bwd, F&& f) {
  for (int64_t b0 = 0; b0 < a.B; b0 += most) {
    f(gn_slice<DT>(a, b0, a.B - b0 < most ? a.B - b0 : most, bwd));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int DT>
hipError_t gn_params_launch(const GnArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((eql_gn_params_kernel<DT>), dim3((unsigned)((a.C + 3) / 4)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

template <int DT, int VEC>
hipError_t gn_fwd_v(const GnArgs& a, hipStream_t stream) {
  auto k = a.act == kActRelu   ? eql_gn_map_kernel<DT, VEC, kActRelu>
           : a.act == kActSilu ? eql_gn_map_kernel<DT, VEC, kActSilu>
           : a.act == kActGelu ? eql_gn_map_kernel<DT, VEC, kActGelu>
                               : eql_gn_map_kernel<DT, VEC, kActNone>;
  const int64_t per = (int64_t)a.chunks * a.cblocks;
  return gn_slices<DT>(a, launch_blocks(256) / per, false, [&](const GnArgs& s) {
    const dim3 n((unsigned)(s.B * per));
    hipLaunchKernelGGL((eql_gn_sums_kernel<DT, VEC>), n, dim3(256), 0, stream, s);
    hipLaunchKernelGGL(k, n, dim3(256), 0, stream, s);
  });
}

template <int DT, int VEC, int ACT>
hipError_t gn_bwd_a(const GnArgs& a, hipStream_t stream) {
  const int64_t per = (int64_t)a.chunks * a.cblocks, tiles = (a.C + 63) / 64, params = (a.C + 3) / 4;
  const int64_t most = (launch_blocks(256) - params) / (per > tiles ? per : tiles);
  const bool whole = a.B <= most;  // the map's last workgroups form dw and db where one launch holds every sequence
  const hipError_t e = gn_slices<DT>(a, most, true, [&](const GnArgs& s) {
    const int64_t n = s.B * per;
    hipLaunchKernelGGL((eql_gn_bsums_kernel<DT, VEC, ACT>), dim3((unsigned)n), dim3(256), 0, stream, s);
    hipLaunchKernelGGL(eql_gn_bchunks_kernel, dim3((unsigned)(s.B * tiles)), dim3(256), 0, stream, s);
    hipLaunchKernelGGL((eql_gn_bmap_kernel<DT, VEC, ACT>), dim3((unsigned)(n + (whole ? params : 0))), dim3(256), 0,
                       stream, s);
  });
  return e != hipSuccess || whole ? e : gn_params_launch<DT>(a, stream);
}
template <int DT, int VEC>
hipError_t gn_bwd_v(const GnArgs& a, hipStream_t stream) {
  if (a.act == kActRelu) return gn_bwd_a<DT, VEC, kActRelu>(a, stream);
  if (a.act == kActSilu) return gn_bwd_a<DT, VEC, kActSilu>(a, stream);
  if (a.act == kActGelu) return gn_bwd_a<DT, VEC, kActGelu>(a, stream);
  return gn_bwd_a<DT, VEC, kActNone>(a, stream);
}

template <int DT, int ACT>
hipError_t gn_hold_a(const GnArgs& a, bool bwd, hipStream_t stream) {
  const hipError_t e = gn_slices<DT>(a, launch_blocks(a.threads) / a.G, bwd, [&](const GnArgs& s) {
    const dim3 n((unsigned)(s.B * a.G));
    if (!bwd) {
      if (a.threads == 256 && a.hold <= 4) hipLaunchKernelGGL((eql_gn_hold_kernel<DT, ACT, 256, 4>), n, dim3(256), 0, stream, s);
      else if (a.threads == 256) hipLaunchKernelGGL((eql_gn_hold_kernel<DT, ACT, 256, 16>), n, dim3(256), 0, stream, s);
      else hipLaunchKernelGGL((eql_gn_hold_kernel<DT, ACT, 1024, 16>), n, dim3(1024), 0, stream, s);
    } else {
      if (a.threads == 256 && a.hold <= 4) hipLaunchKernelGGL((eql_gn_bhold_kernel<DT, ACT, 256, 4>), n, dim3(256), 0, stream, s);
      else if (a.threads == 256) hipLaunchKernelGGL((eql_gn_bhold_kernel<DT, ACT, 256, 16>), n, dim3(256), 0, stream, s);
      else hipLaunchKernelGGL((eql_gn_bhold_kernel<DT, ACT, 512, 16>), n, dim3(512), 0, stream, s);
    }
  });
  return e != hipSuccess || !bwd ? e : gn_params_launch<DT>(a, stream);
}
template <int DT>
hipError_t gn_hold_dt(const GnArgs& a, bool bwd, hipStream_t stream) {
  if (a.act == kActRelu) return gn_hold_a<DT, kActRelu>(a, bwd, stream);
  if (a.act == kActSilu) return gn_hold_a<DT, kActSilu>(a, bwd, stream);
  if (a.act == kActGelu) return gn_hold_a<DT, kActGelu>(a, bwd, stream);
  return gn_hold_a<DT, kActNone>(a, bwd, stream);
}

// Whole 16-byte vectors, or single elements where a row of K is none.
template <int DT>
hipError_t gn_dt(const GnArgs& a, int vec, bool bwd, hipStream_t stream) {
  constexpr int W = DT == kF32 ? 4 : 8;
  if (a.hold) return gn_hold_dt<DT>(a, bwd, stream);
  if (vec == W) return bwd ? gn_bwd_v<DT, W>(a, stream) : gn_fwd_v<DT, W>(a, stream);
  return bwd ? gn_bwd_v<DT, 1>(a, stream) : gn_fwd_v<DT, 1>(a, stream);
}

}  // namespace

hipError_t launch_rotary(int dt, const RotaryArgs& a, int vec, hipStream_t stream) {
  if (dt == kF32) return rotary_dt<kF32>(a, vec, stream);
  if (dt == kF16) return rotary_dt<kF16>(a, vec, stream);
  return rotary_dt<kBF16>(a, vec, stream);
}

// About four workgroups a CU over all sequences (128 images of 3,136 positions: two a CU
// take 20 + 30 us, four 17 + 28), and at least eight positions for each thread where
// there are enough (a thread's start costs as much as several positions).
void gn_plan(GnArgs& a, int vec, int cus, bool bwd) {
  // A group in one workgroup: whole vectors of a group's columns, at most a quarter of
  // the threads, and the fewest threads whose registers hold its rows.
  const int gw = a.K / a.G;
  a.hold = 0;
  if (vec > 1 && gw % vec == 0) {
    const int most = bwd ? 512 : 1024;
    for (int t = 256; t <= most; t = t == 256 ? most : 2 * most) {
      const int vpg = gw / vec;
      if (4 * vpg > t) continue;
      const int64_t r = (a.S + t / vpg - 1) / (t / vpg);
      if (r > 16) continue;
      a.hold = (int)r;
      a.threads = t;
      break;
    }
  }
  const int nv = a.K / vec;
  // vectors that hold whole channels: T / gcd(T, vec) of them, or a multiple
  int whole = a.T;
  for (int v = vec; v > 1 && whole % 2 == 0; v /= 2) whole /= 2;
  a.width = 256 / whole * whole;
  a.cblocks = (nv + a.width - 1) / a.width;
  const int step = nv >= a.width ? 1 : 256 / nv;
  int64_t chunks = (4 * (int64_t)cus + a.B * a.cblocks - 1) / (a.B * a.cblocks);
  const int64_t most = (a.S + 8 * step - 1) / (8 * step);
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  a.rows = (int)((a.S + chunks - 1) / chunks);
  a.chunks = (int)((a.S + a.rows - 1) / a.rows);
}

hipError_t launch_gn_forward(int dt, const GnArgs& a, int vec, hipStream_t stream) {
  if (dt == kF32) return gn_dt<kF32>(a, vec, false, stream);
  if (dt == kF16) return gn_dt<kF16>(a, vec, false, stream);
  return gn_dt<kBF16>(a, vec, false, stream);
}

hipError_t launch_gn_backward(int dt, const GnArgs& a, int vec, hipStream_t stream) {
  if (dt == kF32) return gn_dt<kF32>(a, vec, true, stream);
  if (dt == kF16) return gn_dt<kF16>(a, vec, true, stream);
  return gn_dt<kBF16>(a, vec, true, stream);
}

}  // namespace eqk
