// eql_attn.hip -- windowed attention (eql_attn.h): instantiations, plans and
// launches of one element type (EQK_DT).
#include "eql_attn.h"
#include "eql_launch.h"

namespace eqk {
namespace {

constexpr int DT = EQK_DT;
constexpr int kEB = DT == kF32 ? 4 : 2;

constexpr int row_bytes(int DP) { return (DP == 96 ? 128 : DP) * kEB; }
constexpr int fwd_lds(int DP) { return 2 * (2 * attn_tile(DT) * row_bytes(DP) + 4 * 4); }
constexpr int few_lds(int DP, int keys) { return keys * (2 * attn_fwd_tile(DT, 1) * row_bytes(DP) + 64 * 8); }
constexpr int dkv_lds(int DP) {
  return 2 * (2 * attn_tile(DT) * row_bytes(DP) + 2 * attn_tile(DT) * 4 + 4 * dkv_groups(DT, DP) * 4) +
         (dkv_groups(DT, DP) == 2 ? kAttnDkvKeys * row_bytes(DP) : 0);
}

template <typename K>
hipError_t launch(K k, int64_t blocks, int threads, int lds, hipStream_t stream, const AttnArgs& a) {
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(threads), lds, stream, a);
  return hipGetLastError();
}

template <int DP>
hipError_t fwd(const AttnArgs& a, int waves, hipStream_t stream) {
  const int64_t n = attn_blocks((int64_t)a.B * a.Hkv, (int64_t)((a.R + 32 * waves - 1) / (32 * waves)) * a.parts);
  if constexpr (DT != kF32 || DP <= 64) {
    if (waves == 1 && attn_key_waves(a.parts) == 8)
      return launch(eql_wattn_fwd_kernel<DT, DP, 1, 8>, n, 512, few_lds(DP, 8), stream, a);
    if (waves == 1) return launch(eql_wattn_fwd_kernel<DT, DP, 1, 4>, n, 256, few_lds(DP, 4), stream, a);
  }
  return launch(eql_wattn_fwd_kernel<DT, DP, 4, 1>, n, 256, fwd_lds(DP), stream, a);
}

template <int DP>
hipError_t bwd(const AttnArgs& a, hipStream_t stream) {
  const int64_t nq = attn_blocks((int64_t)a.B * a.Hkv, (a.R + 127) / 128);
  if (nq > 0) {
    const hipError_t e = launch(eql_wattn_dq_kernel<DT, DP, 4>, nq, 256, fwd_lds(DP), stream, a);
    if (e != hipSuccess) return e;
  }
  const int64_t per = (int64_t)a.sink_tiles * a.sink_parts + (int64_t)(a.key_tiles - a.sink_tiles) * a.key_parts;
  if (per == 0) return hipSuccess;
  return launch(eql_wattn_dkv_kernel<DT, DP>, attn_blocks((int64_t)a.B * a.Hkv, per),
                256 * dkv_groups(DT, DP), dkv_lds(DP), stream, a);
}

// The sequences of one launch: fewer than 2^32 threads.
AttnArgs slice(const AttnArgs& a, int b0, int n) {
  AttnArgs s = a;
  auto in = [&](const void* p, const int64_t (&st)[3]) { return p ? (const char*)p + b0 * st[0] * kEB : nullptr; };
  auto out = [&](void* p, const int64_t (&st)[3]) { return p ? (char*)p + b0 * st[0] * kEB : nullptr; };
  s.q = in(a.q, a.qs); s.k = in(a.k, a.ks); s.v = in(a.v, a.vs); s.go = in(a.go, a.gos);
  s.o = out(a.o, a.os); s.dq = out(a.dq, a.dqs); s.dk = out(a.dk, a.dks); s.dv = out(a.dv, a.dvs);
  if (a.lengths) s.lengths = a.lengths + b0;
  if (a.starts) s.starts = a.starts + b0;
  if (a.lse) s.lse = a.lse + (int64_t)b0 * a.Hkv * a.R;
  if (a.delta) s.delta = a.delta + (int64_t)b0 * a.Hkv * a.R;
  s.B = n;
  return s;
}

}  // namespace

template <>
hipError_t wattn_fwd<DT>(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  const int64_t per = attn_blocks(a.Hkv, (int64_t)((a.R + 32 * p.waves - 1) / (32 * p.waves)) * p.parts);
  const int64_t join = p.parts > 1 ? ((int64_t)a.Hkv * a.R * attn_join_waves(p.parts) + 3) / 4 : 0;
  const int64_t most = launch_blocks(512) / (per > join ? per : join);
  if (most < 1) return hipErrorInvalidValue;
  for (int64_t b0 = 0; b0 < a.B; b0 += most) {
    AttnArgs s = slice(a, (int)b0, (int)(a.B - b0 < most ? a.B - b0 : most));
    s.parts = p.parts;
    hipError_t e = a.D <= 32   ? fwd<32>(s, p.waves, stream)
                   : a.D <= 64 ? fwd<64>(s, p.waves, stream)
                   : a.D <= 96 ? fwd<96>(s, p.waves, stream)
                               : fwd<128>(s, p.waves, stream);
    if (e == hipSuccess && p.parts > 1)
      e = launch(eql_wattn_join_kernel<DT>, ((int64_t)s.B * s.Hkv * s.R * attn_join_waves(p.parts) + 3) / 4, 256, 0, stream, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <>
hipError_t wattn_bwd<DT>(const AttnArgs& a, hipStream_t stream) {
  const bool split = a.part != nullptr;
  const int64_t per = (int64_t)a.sink_tiles * a.sink_parts + (int64_t)(a.key_tiles - a.sink_tiles) * a.key_parts;
  const int64_t rows = (a.R + 127) / 128;
  const int64_t tiles = (a.sink_parts > 1 ? a.sink_tiles : 0) + (a.key_parts > 1 ? a.key_tiles - a.sink_tiles : 0);
  const int64_t sums = 2 * tiles * ((kAttnDkvKeys * a.D + 1023) / 1024);  // workgroups that add a head pair's parts
  int64_t grid = attn_blocks(a.Hkv, per > rows ? per : rows);
  if (grid < sums * a.Hkv) grid = sums * a.Hkv;
  const int64_t most = launch_blocks(512) / grid;
  if (most < 1) return hipErrorInvalidValue;
  // (the slices use the same parts, one after another on the stream)
  for (int64_t b0 = 0; b0 < a.B; b0 += most) {
    const AttnArgs s = slice(a, (int)b0, (int)(a.B - b0 < most ? a.B - b0 : most));
    hipError_t e = a.D <= 32   ? bwd<32>(s, stream)
                   : a.D <= 64 ? bwd<64>(s, stream)
                   : a.D <= 96 ? bwd<96>(s, stream)
                               : bwd<128>(s, stream);
    if (e == hipSuccess && split) {
      hipLaunchKernelGGL(eql_wattn_dkv_sum_kernel<DT>, dim3((unsigned)(sums * s.B * s.Hkv)), dim3(256), 0, stream, s,
                         kAttnDkvKeys);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace eqk
