// eql_scan.h -- the selective state space scan, forward and gradients, for gfx950.
//
//   d = softplus(delta + bias);  h_l[n] = exp(d A[n]) h_{l-1}[n] + d b_l[n] x_l;
//   y_l = (sum_n c_l[n] h_l[n] + D x_l) silu(z_l)
// and, with s = dy silu(z), from the last token on
//   g_l[n] = c_l[n] s_l + a_{l+1}[n] g_{l+1}[n],  a = exp(d A)
//   db[n] = sum g d x, dc[n] = sum s h over the columns of a group,  dx = d sum_n g b + D s,
//   dd = sum_n A a g h_{l-1} + x sum_n g b,  dA[n] = sum d a g h_{l-1},  dz = dy (sum_n c h + D x) silu'(z).
//
// A wave takes a block of columns (channel, group element) of one group and walks the tokens in tiles.
// NL lanes share four columns and hold four states of each in registers: a token costs a lane two 16-byte
// reads of d and d x and two of b and c from LDS for 16 states.  Element by element work (softplus, the gate, loads and
// stores in whole vectors) runs on the tile's elements spread over all lanes; d and d x go to the
// scan through LDS, y comes back the same way.  No barrier in the forward: a wave's LDS is its own.
//
// Few columns against many tokens are split into chunks of tokens: one pass forms each chunk's state from
// zero and its sum of d, a small kernel carries the states over the chunks (a chunk multiplies what
// comes in by exp(A sum d)), and the main pass starts every chunk from its own.
#pragma once
#include "eql_common.h"
#include "eql_config.h"
#include "eql_recurrent.h"

namespace eqk {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

// Reads and writes of LDS by lanes of one wave stay in program order; the compiler must keep it.
__device__ __forceinline__ void wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sum over the NL neighbouring lanes that share columns.
template <int NL>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (NL >= 2) v += dpp<0xB1>(v);    // quad_perm 1 0 3 2
  if constexpr (NL >= 4) v += dpp<0x4E>(v);    // quad_perm 2 3 0 1
  if constexpr (NL >= 8) v += dpp<0x141>(v);   // half row mirrored: the other quad
  if constexpr (NL >= 16) v += dpp<0x140>(v);  // row mirrored: the other half
  return v;
}
__device__ __forceinline__ void swap16(float& u, float& v) {  // odd rows of u with even rows of v
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, u), __builtin_bit_cast(unsigned, v), false, false);
  u = __builtin_bit_cast(float, (unsigned)r[0]);
  v = __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ void swap32(float& u, float& v) {  // upper half of u with lower half of v
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, u), __builtin_bit_cast(unsigned, v), false, false);
  u = __builtin_bit_cast(float, (unsigned)r[0]);
  v = __builtin_bit_cast(float, (unsigned)r[1]);
}
// Sums of v0 .. v3 over the lanes with the same place among NL, value r in row r (16 lanes) of the result.
template <int NL>
__device__ __forceinline__ float columns_sum(float v0, float v1, float v2, float v3) {
  swap16(v0, v1);
  swap16(v2, v3);
  float s = v0 + v1, t = v2 + v3;
  swap32(s, t);
  s += t;
  if constexpr (NL <= 1) s += dpp<0x121>(s);  // rows rotated by 1, 2, 4, 8
  if constexpr (NL <= 2) s += dpp<0x122>(s);
  if constexpr (NL <= 4) s += dpp<0x124>(s);
  if constexpr (NL <= 8) s += dpp<0x128>(s);
  return s;
}

// log(1 + e) for 0 <= e <= 1 as 2 atanh(e / (2 + e)), the series to the 13th power: 2e-8 of its value.
__device__ __forceinline__ float log1p_unit(float e) {
  const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
  float p = __builtin_fmaf(q, 1.0f / 13.0f, 1.0f / 11.0f);
  p = __builtin_fmaf(q, p, 1.0f / 9.0f);
  p = __builtin_fmaf(q, p, 1.0f / 7.0f);
  p = __builtin_fmaf(q, p, 1.0f / 5.0f);
  p = __builtin_fmaf(q, p, 1.0f / 3.0f);
  p = __builtin_fmaf(q, p, 1.0f);
  return 2.0f * s * p;
}
__device__ __forceinline__ float softplus(float v) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v));
  return (v > 0.0f ? v : v < 0.0f ? 0.0f : v) + log1p_unit(e);  // NaN stays
}
__device__ __forceinline__ float sigmoid(float v) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  return v < 0.0f ? e * r : r;
}

// Where a wave stands.
struct ScanPlace {
  int64_t b, k;    // sequence, chunk
  int g, blk;      // group, block of its columns
  int col0;        // first column among the padded ones
  int ct0, left;   // first column of the features, columns of the group from it on
  int64_t len;     // tokens that hold data
  int64_t begin, end;
};
template <int NL>
__device__ __forceinline__ ScanPlace scan_place(const ScanArgs& a, int64_t id) {
  ScanPlace p;
  p.blk = (int)(id % a.nblk);
  id /= a.nblk;
  p.g = (int)(id % a.G);
  id /= a.G;
  p.k = id % a.K;
  p.b = id / a.K;
  p.col0 = (p.g * a.nblk + p.blk) * scan_cols(NL);
  p.ct0 = p.g * a.CTg + p.blk * scan_cols(NL);
  p.left = a.CTg - p.blk * scan_cols(NL);
  p.len = a.lengths ? min(max((int64_t)a.lengths[p.b], (int64_t)0), a.L) : a.L;
  p.begin = p.k * a.chunk;
  p.end = min(p.begin + a.chunk, a.L);
  return p;
}

// The lane's elements of a tile of [TT][CH]: NV vectors of VEC, vector v at token tok(v), column at.
template <int DT, int NL>
struct ScanTile {
  static constexpr int CH = scan_cols(NL), TT = scan_tile(NL), EPT = scan_ept(NL), VEC = scan_vec(DT, NL);
  static constexpr int NV = EPT / VEC, VT = CH / VEC, EB = DT == kF32 ? 4 : 2;
  static constexpr int W = VEC * EB / 4;  // 32-bit words of a vector
  static constexpr int NP = 4 * NL;
  static constexpr int NBC = (TT * NP + 63) / 64;  // elements of b, and of c, that a lane loads
  using E = typename Elem<DT>::T;
  struct Raw {
    uint32_t w[NV * W];
  };
  static __device__ __forceinline__ int at() { return (threadIdx.x & 63) % VT * VEC; }
  static __device__ __forceinline__ int tok(int v) { return v * (64 / VT) + (threadIdx.x & 63) / VT; }

  template <bool WHOLE>
  static __device__ __forceinline__ void load(Raw& r, const void* base, int64_t stride, int nt, int left) {
    const E* p = reinterpret_cast<const E*>(base);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int t = tok(v);
      const bool on = t < nt;
      const E* q = p + t * stride + at();
      if constexpr (WHOLE) {
        const bool ok = on && at() < left;
        if constexpr (W == 4) {
          const u32x4 x = ok ? *reinterpret_cast<const u32x4*>(q) : u32x4{0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < 4; ++i) r.w[v * W + i] = x[i];
        } else {
          const u32x2 x = ok ? *reinterpret_cast<const u32x2*>(q) : u32x2{0, 0};
#pragma unroll
          for (int i = 0; i < W; ++i) r.w[v * W + i] = x[i];
        }
      } else if constexpr (EB == 4) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          r.w[v * W + i] = on && at() + i < left ? __builtin_bit_cast(uint32_t, q[i]) : 0u;
      } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const uint32_t lo = on && at() + 2 * i < left ? h[2 * i] : 0u, hi = on && at() + 2 * i + 1 < left ? h[2 * i + 1] : 0u;
          r.w[v * W + i] = lo | hi << 16;
        }
      }
    }
  }
  static __device__ __forceinline__ void floats(const Raw& r, float (&f)[EPT]) { raw_to_floats<DT, NV * W>(r.w, f); }

  // stores the elements of tokens below `rows`
  template <bool WHOLE>
  static __device__ __forceinline__ void store(const float (&f)[EPT], void* base, int64_t stride, int rows, int left) {
    E* p = reinterpret_cast<E*>(base);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int t = tok(v);
      if (t >= rows) continue;
      E* q = p + t * stride + at();
      if constexpr (WHOLE) {
        if (at() >= left) continue;
        uint32_t w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = pack2<DT>(f[v * VEC + i * (4 / EB)], f[v * VEC + i * (4 / EB) + (EB == 2)]);
        if constexpr (W == 4) *reinterpret_cast<u32x4*>(q) = u32x4{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<u32x2*>(q) = u32x2{w[0], w[1]};
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (at() + i < left) q[i] = (E)f[v * VEC + i];
      }
    }
  }
  // the tile [TT][CH] of LDS
  static __device__ __forceinline__ void put(float* tile, const float (&f)[EPT]) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < VEC; i += 4)
        *reinterpret_cast<floatx4*>(tile + tok(v) * CH + at() + i) =
            floatx4{f[v * VEC + i], f[v * VEC + i + 1], f[v * VEC + i + 2], f[v * VEC + i + 3]};
  }
  static __device__ __forceinline__ void get(const float* tile, float (&f)[EPT]) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < VEC; i += 4) {
        const floatx4 q = *reinterpret_cast<const floatx4*>(tile + tok(v) * CH + at() + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[v * VEC + i + j] = q[j];
      }
  }
  // b or c of a tile: element i * 64 + lane of [TT][NP]
  struct Bc {
    E e[NBC];
  };
  static __device__ __forceinline__ void load_bc(Bc& r, const void* base, int64_t stride, int nt, int N) {
    const E* p = reinterpret_cast<const E*>(base);
#pragma unroll
    for (int i = 0; i < NBC; ++i) {
      const int j = i * 64 + (threadIdx.x & 63), t = j / NP, n = j % NP;
      r.e[i] = t < nt && n < N ? p[t * stride + n] : (E)0.0f;
    }
  }
  static __device__ __forceinline__ void put_bc(float* tile, const Bc& r) {
#pragma unroll
    for (int i = 0; i < NBC; ++i) {
      const int j = i * 64 + (threadIdx.x & 63);
      if (TT * NP >= 64 || j < TT * NP) tile[j] = (float)r.e[i];
    }
  }
};

// A of the lane's four columns and four states, times log2(e); 0 outside, where a state stays 0.
template <int NL>
__device__ __forceinline__ void scan_decay(const ScanArgs& a, const ScanPlace& p, float (&A2)[4][4]) {
  const int lane = threadIdx.x & 63, n0 = lane % NL * 4, c0 = lane / NL * 4;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const bool ok = c0 + q < p.left && n0 + n < a.N;
      A2[q][n] = ok ? a.A[(int64_t)((p.ct0 + c0 + q) / a.T) * a.N + n0 + n] * kLog2e : 0.0f;
    }
}
// The lane's states in [cols][NP] (whole) or [CT][N].
template <int NL>
__device__ __forceinline__ void load_padded(const float* base, float (&h)[4][4]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(base + (lane / NL * 4 + q) * (4 * NL) + lane % NL * 4);
#pragma unroll
    for (int n = 0; n < 4; ++n) h[q][n] = v[n];
  }
}
template <int NL>
__device__ __forceinline__ void store_padded(float* base, const float (&h)[4][4]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<floatx4*>(base + (lane / NL * 4 + q) * (4 * NL) + lane % NL * 4) =
        floatx4{h[q][0], h[q][1], h[q][2], h[q][3]};
}
template <int NL>
__device__ __forceinline__ void load_state(const ScanArgs& a, const ScanPlace& p, const float* base, float (&h)[4][4]) {
  const int lane = threadIdx.x & 63, n0 = lane % NL * 4, c0 = lane / NL * 4;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float* s = base + (p.b * a.CT + p.ct0 + c0 + q) * a.N + n0;
    if (c0 + q < p.left && a.N == 4 * NL && ((uintptr_t)base & 15) == 0) {
      const floatx4 v = *reinterpret_cast<const floatx4*>(s);
#pragma unroll
      for (int n = 0; n < 4; ++n) h[q][n] = v[n];
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) h[q][n] = c0 + q < p.left && n0 + n < a.N ? s[n] : 0.0f;
    }
  }
}
template <int NL>
__device__ __forceinline__ void store_state(const ScanArgs& a, const ScanPlace& p, float* base, const float (&h)[4][4]) {
  const int lane = threadIdx.x & 63, n0 = lane % NL * 4, c0 = lane / NL * 4;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (c0 + q >= p.left) continue;
    float* s = base + (p.b * a.CT + p.ct0 + c0 + q) * a.N + n0;
    if (a.N == 4 * NL && ((uintptr_t)base & 15) == 0) {
      *reinterpret_cast<floatx4*>(s) = floatx4{h[q][0], h[q][1], h[q][2], h[q][3]};
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n0 + n < a.N) s[n] = h[q][n];
    }
  }
}
// The parameter of the channels of the lane's vector, v where p is NULL.
template <int VEC>
__device__ __forceinline__ void scan_param(const ScanArgs& a, const ScanPlace& p, const float* src, int at, float (&f)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) f[i] = src && at + i < p.left ? src[(p.ct0 + at + i) / a.T] : 0.0f;
}

// One token: a = exp(d A), h = a h + (d x) b.
__device__ __forceinline__ void scan_step(float (&h)[4][4], const float (&A2)[4][4], const floatx4& d, const floatx4& dx,
                                          const floatx4& bb) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n)
      h[q][n] = __builtin_fmaf(__builtin_amdgcn_exp2f(d[q] * A2[q][n]), h[q][n], dx[q] * bb[n]);
}

// ---- forward ---------------------------------------------------------------
// STATES: only the state that a chunk forms from zero and its sum of d (chunks 0 .. K - 2).
template <int NL>
constexpr int scan_fwd_lds() {  // floats of a wave
  return 2 * scan_tile(NL) * scan_cols(NL) + 2 * scan_tile(NL) * 4 * NL;
}
template <int DT, int NL, bool WHOLE, bool STATES>
__global__ __launch_bounds__(64 * kScanWaves) void eql_scan_fwd_kernel(const ScanArgs a) {
  using TL = ScanTile<DT, NL>;
  constexpr int TT = TL::TT, CH = TL::CH, EPT = TL::EPT, VEC = TL::VEC, NP = TL::NP, EB = TL::EB;
  __shared__ __attribute__((aligned(16))) float lds[kScanWaves * scan_fwd_lds<NL>()];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = (a.first + blockIdx.x) * kScanWaves + wave;
  if (id >= a.B * a.K * a.G * a.nblk) return;  // (no barrier follows)
  const ScanPlace p = scan_place<NL>(a, id);
  if (STATES && p.k == a.K - 1) return;
  float* const ds = lds + wave * scan_fwd_lds<NL>();
  float* const us = ds + TT * CH;
  float* const bs = us + TT * CH;
  float* const cs = bs + TT * NP;
  const int n0 = lane % NL * 4, c0 = lane / NL * 4, at = TL::at();
  float A2[4][4], h[4][4], bias[VEC], skip[VEC], total[4] = {0.f, 0.f, 0.f, 0.f};
  scan_decay<NL>(a, p, A2);
  scan_param<VEC>(a, p, a.bias, at, bias);
  if constexpr (!STATES) scan_param<VEC>(a, p, a.D, at, skip);
  const int64_t slot = (p.b * a.K + p.k) * a.cols + p.col0;
  if (!STATES && a.K > 1) load_padded<NL>(a.carry + slot * NP, h);
  else if (!STATES && a.h0) load_state<NL>(a, p, a.h0, h);
  else
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int n = 0; n < 4; ++n) h[q][n] = 0.0f;
  const int64_t stop = min(p.len, p.end);
  // addresses of the wave's first token and column
  auto base = [&](const void* q, const int64_t (&st)[2], int64_t l) { return (const char*)q + (p.b * st[0] + l * st[1] + p.ct0) * EB; };
  auto bcbase = [&](const void* q, const int64_t (&st)[3], int64_t l) { return (const char*)q + (p.b * st[0] + l * st[1] + p.g * st[2]) * EB; };
  typename TL::Raw xr, dr, zr;
  typename TL::Bc br, cr;
  auto fetch = [&](int64_t l0) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    TL::template load<WHOLE>(xr, base(a.x, a.xs, l0), a.xs[1], nt, p.left);
    TL::template load<WHOLE>(dr, base(a.delta, a.ds, l0), a.ds[1], nt, p.left);
    TL::load_bc(br, bcbase(a.b, a.bs, l0), a.bs[1], nt, a.N);
    if constexpr (!STATES) {
      if (a.z) TL::template load<WHOLE>(zr, base(a.z, a.zs, l0), a.zs[1], nt, p.left);
      TL::load_bc(cr, bcbase(a.c, a.cs, l0), a.cs[1], nt, a.N);
    }
  };
  if (p.begin < stop) fetch(p.begin);
  for (int64_t l0 = p.begin; l0 < stop; l0 += TT) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    float xf[EPT], df[EPT], zf[EPT];
    TL::floats(xr, xf);
    TL::floats(dr, df);
    if constexpr (!STATES) {
      if (a.z) TL::floats(zr, zf);
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      df[e] += bias[e % VEC];
      if (a.softplus) df[e] = softplus(df[e]);
      if (TL::tok(e / VEC) >= nt) df[e] = 0.0f;
    }
    wave_order();  // the tile before has been read
    TL::put(ds, df);
#pragma unroll
    for (int e = 0; e < EPT; ++e) df[e] = TL::tok(e / VEC) >= nt ? 0.0f : df[e] * xf[e];
    TL::put(us, df);
    TL::put_bc(bs, br);
    if constexpr (!STATES) TL::put_bc(cs, cr);
    if (l0 + TT < stop) fetch(l0 + TT);
    if constexpr (!STATES)
      if (a.states) store_padded<NL>(a.states + ((p.b * a.tiles + l0 / TT) * a.cols + p.col0) * NP, h);
    wave_order();
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int t = 0; t < TT; ++t) {
      const floatx4 d = *reinterpret_cast<const floatx4*>(ds + t * CH + c0), u = *reinterpret_cast<const floatx4*>(us + t * CH + c0);
      const floatx4 bb = *reinterpret_cast<const floatx4*>(bs + t * NP + n0);
      scan_step(h, A2, d, u, bb);
      if constexpr (STATES) {
#pragma unroll
        for (int q = 0; q < 4; ++q) part[q] += d[q];
      } else {
        const floatx4 cc = *reinterpret_cast<const floatx4*>(cs + t * NP + n0);
        floatx4 y;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float s = h[q][0] * cc[0];
#pragma unroll
          for (int n = 1; n < 4; ++n) s = __builtin_fmaf(h[q][n], cc[n], s);
          y[q] = lanes_sum<NL>(s);
        }
        // in place of d x, which every lane of these columns has read
        if (lane % NL == 0) *reinterpret_cast<floatx4*>(us + t * CH + c0) = y;
      }
    }
    if constexpr (STATES) {
#pragma unroll
      for (int q = 0; q < 4; ++q) total[q] += part[q];
    } else {
      wave_order();
      float yf[EPT];
      TL::get(us, yf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        yf[e] = __builtin_fmaf(skip[e % VEC], xf[e], yf[e]);
        if (a.z) yf[e] *= zf[e] * sigmoid(zf[e]);
        if (TL::tok(e / VEC) >= nt) yf[e] = 0.0f;
      }
      TL::template store<WHOLE>(yf, (char*)a.y + ((p.b * a.L + l0) * a.CT + p.ct0) * EB, a.CT, (int)min(p.end - l0, (int64_t)TT), p.left);
    }
  }
  if constexpr (STATES) {
    store_padded<NL>(a.carry + slot * NP, h);
    if (lane % NL == 0) *reinterpret_cast<floatx4*>(a.sums + slot + c0) = floatx4{total[0], total[1], total[2], total[3]};
  } else {
    float zero[EPT];
#pragma unroll
    for (int e = 0; e < EPT; ++e) zero[e] = 0.0f;
    const int64_t from = p.begin + (max(stop - p.begin, (int64_t)0) + TT - 1) / TT * TT;  // tiles of padding alone
    for (int64_t l0 = from; l0 < p.end; l0 += TT)
      TL::template store<WHOLE>(zero, (char*)a.y + ((p.b * a.L + l0) * a.CT + p.ct0) * EB, a.CT, (int)min(p.end - l0, (int64_t)TT), p.left);
    if (a.hT && p.k == a.K - 1) store_state<NL>(a, p, a.hT, h);
  }
}

// Carries the states over the chunks of a sequence, in place: what a chunk formed from zero becomes what it
// starts from.  BACK: from the last chunk to the first, the gradient behind a chunk.  A thread takes one column's state.
template <bool BACK>
__global__ __launch_bounds__(256) void eql_scan_carry_kernel(const ScanArgs a, int NP) {
  const int64_t i = (a.first + blockIdx.x) * 256 + threadIdx.x, per = (int64_t)a.cols * NP;
  if (i >= a.B * per) return;
  const int64_t b = i / per;
  const int col = (int)(i % per / NP), n = (int)(i % NP);
  const int CH = 1024 / NP;  // columns of a wave's block
  const int g = col / (a.nblk * CH), in = col - g * a.nblk * CH;
  const bool real = in < a.CTg && n < a.N;
  const int ct = g * a.CTg + in;
  const float A2 = real ? a.A[(int64_t)(ct / a.T) * a.N + n] * kLog2e : 0.0f;
  const float* first = BACK ? a.dhT : a.h0;
  float h = first && real ? first[(b * a.CT + ct) * a.N + n] : 0.0f;
  float* c = a.carry + (b * a.K * a.cols + col) * NP + n;
  const float* s = a.sums + b * a.K * a.cols + col;
  const int64_t cstep = (int64_t)a.cols * NP;
  // the first chunk of the way has nothing before it; the last one's own result is not wanted
  float v = c[(BACK ? a.K - 1 : 0) * cstep], d = s[(int64_t)(BACK ? a.K - 1 : 0) * a.cols];
  for (int j = 0; j < a.K - 1; ++j) {
    const int64_t k = BACK ? a.K - 1 - j : j, next = BACK ? k - 1 : k + 1;
    const bool more = j + 1 < a.K - 1;
    const float v1 = more ? c[next * cstep] : 0.0f, d1 = more ? s[next * a.cols] : 0.0f;
    c[k * cstep] = h;
    h = __builtin_fmaf(__builtin_amdgcn_exp2f(d * A2), h, v);
    v = v1;
    d = d1;
  }
  c[(BACK ? 0 : a.K - 1) * cstep] = h;
}

// ---- gradients ---------------------------------------------------------------
// r behind a chunk from zero, and its sum of d (chunks 1 .. K - 1): r = a (c s + r) from the last token to the first.
template <int DT, int NL, bool WHOLE>
__global__ __launch_bounds__(64 * kScanWaves) void eql_scan_back_kernel(const ScanArgs a) {
  using TL = ScanTile<DT, NL>;
  constexpr int TT = TL::TT, CH = TL::CH, EPT = TL::EPT, VEC = TL::VEC, NP = TL::NP, EB = TL::EB;
  __shared__ __attribute__((aligned(16))) float lds[kScanWaves * scan_fwd_lds<NL>()];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = (a.first + blockIdx.x) * kScanWaves + wave;
  if (id >= a.B * a.K * a.G * a.nblk) return;  // (no barrier follows)
  const ScanPlace p = scan_place<NL>(a, id);
  if (p.k == 0) return;
  float* const ds = lds + wave * scan_fwd_lds<NL>();
  float* const ss = ds + TT * CH;
  float* const cs = ss + TT * CH;
  const int n0 = lane % NL * 4, c0 = lane / NL * 4, at = TL::at();
  float A2[4][4], r[4][4], bias[VEC], total[4] = {0.f, 0.f, 0.f, 0.f};
  scan_decay<NL>(a, p, A2);
  scan_param<VEC>(a, p, a.bias, at, bias);
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) r[q][n] = 0.0f;
  const int64_t stop = min(p.len, p.end);
  auto base = [&](const void* q, const int64_t (&st)[2], int64_t l) { return (const char*)q + (p.b * st[0] + l * st[1] + p.ct0) * EB; };
  typename TL::Raw yr, dr, zr;
  typename TL::Bc cr;
  auto fetch = [&](int64_t l0) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    TL::template load<WHOLE>(yr, (const char*)a.dy + ((p.b * a.L + l0) * a.CT + p.ct0) * EB, a.CT, nt, p.left);
    TL::template load<WHOLE>(dr, base(a.delta, a.ds, l0), a.ds[1], nt, p.left);
    if (a.z) TL::template load<WHOLE>(zr, base(a.z, a.zs, l0), a.zs[1], nt, p.left);
    TL::load_bc(cr, (const char*)a.c + (p.b * a.cs[0] + l0 * a.cs[1] + p.g * a.cs[2]) * EB, a.cs[1], nt, a.N);
  };
  const int64_t tiles = (max(stop - p.begin, (int64_t)0) + TT - 1) / TT;
  if (tiles > 0) fetch(p.begin + (tiles - 1) * TT);
  for (int64_t tile = tiles - 1; tile >= 0; --tile) {
    const int64_t l0 = p.begin + tile * TT;
    const int nt = (int)min(stop - l0, (int64_t)TT);
    float sf[EPT], df[EPT], zf[EPT];
    TL::floats(yr, sf);
    TL::floats(dr, df);
    if (a.z) {
      TL::floats(zr, zf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) sf[e] *= zf[e] * sigmoid(zf[e]);
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      df[e] += bias[e % VEC];
      if (a.softplus) df[e] = softplus(df[e]);
      if (TL::tok(e / VEC) >= nt) df[e] = sf[e] = 0.0f;
    }
    wave_order();
    TL::put(ds, df);
    TL::put(ss, sf);
    TL::put_bc(cs, cr);
    if (tile > 0) fetch(l0 - TT);
    wave_order();
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int t = TT - 1; t >= 0; --t) {
      const floatx4 d = *reinterpret_cast<const floatx4*>(ds + t * CH + c0), s = *reinterpret_cast<const floatx4*>(ss + t * CH + c0);
      const floatx4 cc = *reinterpret_cast<const floatx4*>(cs + t * NP + n0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        part[q] += d[q];
#pragma unroll
        for (int n = 0; n < 4; ++n)
          r[q][n] = __builtin_amdgcn_exp2f(d[q] * A2[q][n]) * __builtin_fmaf(cc[n], s[q], r[q][n]);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) total[q] += part[q];
  }
  const int64_t slot = (p.b * a.K + p.k) * a.cols + p.col0;
  store_padded<NL>(a.carry + slot * NP, r);
  if (lane % NL == 0) *reinterpret_cast<floatx4*>(a.sums + slot + c0) = floatx4{total[0], total[1], total[2], total[3]};
}

// The gradients.  The waves of a workgroup take neighbouring column blocks of one group and chunk, so that db
// and dc are summed over them before they leave; a tile is walked from its last run of SUB tokens to the
// first: the states of a run are formed again from the tile's first one and kept in registers.
template <int NL>
constexpr int scan_bwd_lds() {  // floats of a wave
  return 3 * scan_tile(NL) * scan_cols(NL) + 2 * scan_tile(NL) * 4 * NL;
}
template <int NL>
constexpr int scan_red_lds() {  // floats of a wave's db and dc, twice
  return 2 * 2 * scan_tile(NL) * 4 * NL;
}
template <int NL>
constexpr int scan_bwd_bytes(int waves) {
  return waves * (scan_bwd_lds<NL>() + scan_red_lds<NL>()) * 4;
}
template <int DT, int NL, bool WHOLE, int SUB>
__global__ __launch_bounds__(64 * kScanWaves, SUB > 8 ? 1 : 2) void eql_scan_bwd_kernel(const ScanArgs a, int waves) {
  using TL = ScanTile<DT, NL>;
  constexpr int TT = TL::TT, CH = TL::CH, EPT = TL::EPT, VEC = TL::VEC, NP = TL::NP, EB = TL::EB;
  using E = typename TL::E;
  extern __shared__ __attribute__((aligned(16))) float smem[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // workgroup: (sequence, chunk, group, run of `waves` blocks)
  int64_t id = a.first + blockIdx.x;
  const int run = (int)(id % a.P);
  id /= a.P;
  const bool on = run * waves + wave < a.nblk;
  ScanPlace p = scan_place<NL>(a, id * a.nblk + min(run * waves + wave, a.nblk - 1));
  if (!on) p.left = 0;
  float* const ds = smem + wave * scan_bwd_lds<NL>();
  float* const us = ds + TT * CH;
  float* const ss = us + TT * CH;
  float* const bs = ss + TT * CH;
  float* const cs = bs + TT * NP;
  float* const red = smem + waves * scan_bwd_lds<NL>();  // [2][waves][TT][2][NP]
  const int n0 = lane % NL * 4, c0 = lane / NL * 4, at = TL::at();
  float A2[4][4], g[4][4], dA[4][4], bias[VEC], skip[VEC], dskip[VEC], dbias[VEC];
  scan_decay<NL>(a, p, A2);
  scan_param<VEC>(a, p, a.bias, at, bias);
  scan_param<VEC>(a, p, a.D, at, skip);
#pragma unroll
  for (int i = 0; i < VEC; ++i) dskip[i] = dbias[i] = 0.0f;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) g[q][n] = dA[q][n] = 0.0f;
  const int64_t slot = (p.b * a.K + p.k) * a.cols + p.col0;
  if (a.K > 1 && on) load_padded<NL>(a.carry + slot * NP, g);
  else if (a.dhT) load_state<NL>(a, p, a.dhT, g);
  const int64_t stop = min(p.len, p.end);
  auto base = [&](const void* q, const int64_t (&st)[2], int64_t l) { return (const char*)q + (p.b * st[0] + l * st[1] + p.ct0) * EB; };
  auto dense = [&](const void* q, int64_t l) { return (char*)q + ((p.b * a.L + l) * a.CT + p.ct0) * EB; };
  auto bcbase = [&](const void* q, const int64_t (&st)[3], int64_t l) { return (const char*)q + (p.b * st[0] + l * st[1] + p.g * st[2]) * EB; };
  const int64_t tiles = (max(stop - p.begin, (int64_t)0) + TT - 1) / TT;
  float* const part = a.part + (p.b * a.K + p.k) * (a.N + 2) * a.cols + p.col0;
  int odd = 0, turns = 0;
  bool flushed = false;
  auto flush = [&] {  // the lane's sums of dA to memory
    if (!on) return;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if (n0 + n >= a.N) continue;
      floatx4* const q = reinterpret_cast<floatx4*>(part + (int64_t)(n0 + n) * a.cols + c0);
      floatx4 v = floatx4{dA[0][n], dA[1][n], dA[2][n], dA[3][n]};
      if (flushed) v += *q;
      *q = v;
    }
    flushed = true;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int n = 0; n < 4; ++n) dA[q][n] = 0.0f;
  };
  for (int64_t tile = tiles - 1; tile >= 0; --tile, odd ^= 1) {
    const int64_t l0 = p.begin + tile * TT;
    const int nt = (int)min(stop - l0, (int64_t)TT);
    // the tile's elements: read here for the scan and again, from the caches, for what follows it
    typename TL::Raw xr, dr, zr, yr;
    auto fetch = [&] {
      TL::template load<WHOLE>(xr, base(a.x, a.xs, l0), a.xs[1], nt, p.left);
      TL::template load<WHOLE>(dr, base(a.delta, a.ds, l0), a.ds[1], nt, p.left);
      TL::template load<WHOLE>(yr, dense(a.dy, l0), a.CT, nt, p.left);
      if (a.z) TL::template load<WHOLE>(zr, base(a.z, a.zs, l0), a.zs[1], nt, p.left);
    };
    fetch();
    {
      float xf[EPT], df[EPT], sf[EPT];
      TL::floats(xr, xf);
      TL::floats(dr, df);
      TL::floats(yr, sf);
      if (a.z) {
        float zf[EPT];
        TL::floats(zr, zf);
#pragma unroll
        for (int e = 0; e < EPT; ++e) sf[e] *= zf[e] * sigmoid(zf[e]);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        df[e] += bias[e % VEC];
        if (a.softplus) df[e] = softplus(df[e]);
        if (TL::tok(e / VEC) >= nt) df[e] = sf[e] = 0.0f;
        dskip[e % VEC] = __builtin_fmaf(sf[e], xf[e], dskip[e % VEC]);
      }
      typename TL::Bc br, cr;
      TL::load_bc(br, bcbase(a.b, a.bs, l0), a.bs[1], nt, a.N);
      TL::load_bc(cr, bcbase(a.c, a.cs, l0), a.cs[1], nt, a.N);
      wave_order();
      TL::put(ds, df);
      TL::put(ss, sf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) df[e] = TL::tok(e / VEC) >= nt ? 0.0f : df[e] * xf[e];
      TL::put(us, df);
      TL::put_bc(bs, br);
      TL::put_bc(cs, cr);
    }
    wave_order();
    float* const mine = red + ((odd * waves + wave) * TT * 2) * NP;
    const float* const start = a.states + ((p.b * a.tiles + l0 / TT) * a.cols + p.col0) * NP;
#pragma unroll 1
    for (int s0 = TT - SUB; s0 >= 0; s0 -= SUB) {
      float h[4][4] = {}, H[SUB][4][4];  // H[i]: the state before token s0 + i
      if (on) load_padded<NL>(start, h);
#pragma unroll 4
      for (int t = 0; t < s0; ++t)
        scan_step(h, A2, *reinterpret_cast<const floatx4*>(ds + t * CH + c0), *reinterpret_cast<const floatx4*>(us + t * CH + c0),
                  *reinterpret_cast<const floatx4*>(bs + t * NP + n0));
#pragma unroll
      for (int i = 0; i < SUB; ++i) {
        const int t = s0 + i;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int n = 0; n < 4; ++n) H[i][q][n] = h[q][n];
        scan_step(h, A2, *reinterpret_cast<const floatx4*>(ds + t * CH + c0), *reinterpret_cast<const floatx4*>(us + t * CH + c0),
                  *reinterpret_cast<const floatx4*>(bs + t * NP + n0));
        __builtin_amdgcn_sched_barrier(0);
      }
      // the way back reads the tokens and forms the exponentials again: kept, they would take as many registers
      // as the states
      asm volatile("" ::: "memory");
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int n = 0; n < 4; ++n) asm volatile("" : "+v"(A2[q][n]));
#pragma unroll
      for (int i = SUB - 1; i >= 0; --i) {
        const int t = s0 + i;
        const floatx4 d = *reinterpret_cast<const floatx4*>(ds + t * CH + c0), u = *reinterpret_cast<const floatx4*>(us + t * CH + c0);
        const floatx4 s = *reinterpret_cast<const floatx4*>(ss + t * CH + c0);
        const floatx4 bb = *reinterpret_cast<const floatx4*>(bs + t * NP + n0), cc = *reinterpret_cast<const floatx4*>(cs + t * NP + n0);
        float db[4] = {0.f, 0.f, 0.f, 0.f}, dc[4] = {0.f, 0.f, 0.f, 0.f};
        floatx4 gb, ga, ch;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float sb = 0.0f, sa = 0.0f, sc = 0.0f;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float now = i + 1 < SUB ? H[i + 1 < SUB ? i + 1 : i][q][n] : h[q][n];  // the state after token t
            g[q][n] = __builtin_fmaf(cc[n], s[q], g[q][n]);
            dc[n] = __builtin_fmaf(s[q], now, dc[n]);
            sc = __builtin_fmaf(cc[n], now, sc);
            db[n] = __builtin_fmaf(g[q][n], u[q], db[n]);
            sb = __builtin_fmaf(g[q][n], bb[n], sb);
            g[q][n] *= __builtin_amdgcn_exp2f(d[q] * A2[q][n]);
            const float m = g[q][n] * H[i][q][n];
            sa = __builtin_fmaf(A2[q][n], m, sa);
            dA[q][n] = __builtin_fmaf(d[q], m, dA[q][n]);
          }
          gb[q] = lanes_sum<NL>(sb);
          ga[q] = lanes_sum<NL>(sa);
          ch[q] = lanes_sum<NL>(sc);
        }
        // d, d x and s of this token have been read by every lane of these columns
        if (lane % NL == 0) {
          *reinterpret_cast<floatx4*>(us + t * CH + c0) = gb;
          *reinterpret_cast<floatx4*>(ds + t * CH + c0) = ga;
          *reinterpret_cast<floatx4*>(ss + t * CH + c0) = ch;
        }
        const float rb = columns_sum<NL>(db[0], db[1], db[2], db[3]), rc = columns_sum<NL>(dc[0], dc[1], dc[2], dc[3]);
        if (lane % 16 < NL) {  // state n0 + row
          mine[(t * 2) * NP + n0 + lane / 16] = rb;
          mine[(t * 2 + 1) * NP + n0 + lane / 16] = rc;
        }
        __builtin_amdgcn_sched_barrier(0);  // bounds what is read ahead: the states take the registers
      }
    }
    if (++turns == 32) {  // sums of no more than 32 tiles in registers, so that long ones lose no digits
      turns = 0;
      flush();
    }
    wave_order();
    fetch();
    {
      float xf[EPT], df[EPT], sf[EPT], f[EPT], o[EPT];
      TL::floats(xr, xf);
      TL::floats(dr, df);
      TL::floats(yr, sf);
      TL::get(us, f);  // sum_n g b
      const int rows = (int)min(p.end - l0, (int64_t)TT);
      if (a.z) {
        float zf[EPT], ch[EPT];
        TL::floats(zr, zf);
        TL::get(ss, ch);
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
          const float sg = sigmoid(zf[e]), y0 = __builtin_fmaf(skip[e % VEC], xf[e], ch[e]);
          ch[e] = TL::tok(e / VEC) >= nt ? 0.0f : sf[e] * y0 * sg * __builtin_fmaf(zf[e], 1.0f - sg, 1.0f);
          sf[e] *= zf[e] * sg;
        }
        if (a.dz) TL::template store<WHOLE>(ch, dense(a.dz, l0), a.CT, rows, p.left);
      }
      TL::get(ds, o);  // sum_n A a g h, times log2(e)
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        const bool in = TL::tok(e / VEC) < nt;
        const float v = df[e] + bias[e % VEC];
        const float d = a.softplus ? softplus(v) : v, dd = __builtin_fmaf(kLn2, o[e], xf[e] * f[e]);
        const float dv = a.softplus ? dd * sigmoid(v) : dd;
        o[e] = in ? dv : 0.0f;
        dbias[e % VEC] += o[e];
        f[e] = in ? __builtin_fmaf(skip[e % VEC], sf[e], d * f[e]) : 0.0f;
      }
      TL::template store<WHOLE>(o, dense(a.ddelta, l0), a.CT, rows, p.left);
      TL::template store<WHOLE>(f, dense(a.dx, l0), a.CT, rows, p.left);
    }
    __syncthreads();  // (every wave of the workgroup walks the same tiles)
    for (int i = threadIdx.x; i < nt * 2 * NP; i += 64 * waves) {
      float v = red[odd * waves * TT * 2 * NP + i];
      for (int w = 1; w < waves; ++w) v += red[(odd * waves + w) * TT * 2 * NP + i];
      const int t = i / (2 * NP), j = i % (2 * NP);
      const int64_t at_bc = (p.b * a.L + l0 + t) * a.G + p.g;
      if (a.P > 1) a.bcpart[(at_bc * a.P + run) * 2 * NP + j] = v;
      else if (j % NP < a.N) reinterpret_cast<E*>(j < NP ? a.db : a.dc)[at_bc * a.N + j % NP] = (E)v;
    }
  }
  // padding behind the sequence
  {
    float zero[EPT];
#pragma unroll
    for (int e = 0; e < EPT; ++e) zero[e] = 0.0f;
    for (int64_t l0 = p.begin + tiles * TT; l0 < p.end; l0 += TT) {
      const int rows = (int)min(p.end - l0, (int64_t)TT);
      TL::template store<WHOLE>(zero, dense(a.dx, l0), a.CT, rows, p.left);
      TL::template store<WHOLE>(zero, dense(a.ddelta, l0), a.CT, rows, p.left);
      if (a.dz) TL::template store<WHOLE>(zero, dense(a.dz, l0), a.CT, rows, p.left);
    }
    if (a.P == 1) {
      const int64_t from = max(p.begin, stop), n = max(p.end - from, (int64_t)0) * a.N;
      for (int64_t i = threadIdx.x; i < n; i += 64 * waves) {
        const int64_t o = ((p.b * a.L + from + i / a.N) * a.G + p.g) * a.N + i % a.N;
        reinterpret_cast<E*>(a.db)[o] = (E)0.0f;
        reinterpret_cast<E*>(a.dc)[o] = (E)0.0f;
      }
    }
  }
  if (a.dh0 && p.k == 0) store_state<NL>(a, p, a.dh0, g);
  if (!on) return;
  flush();
  // lanes with the same columns lie VT apart
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
#pragma unroll
    for (int d = TL::VT; d < 64; d *= 2) {
      dskip[i] += __shfl_xor(dskip[i], d);
      dbias[i] += __shfl_xor(dbias[i], d);
    }
    if (lane < TL::VT) {
      part[(int64_t)a.N * a.cols + at + i] = dskip[i];
      part[(int64_t)(a.N + 1) * a.cols + at + i] = dbias[i];
    }
  }
}

// db and dc: the parts of a token's P workgroups in order.
template <int DT>
__global__ __launch_bounds__(256) void eql_scan_bc_kernel(const ScanArgs a, int NP) {
  using E = typename Elem<DT>::T;
  const int64_t i = (a.first + blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.B * a.L * a.G * 2 * NP) return;
  const int64_t at = i / (2 * NP), l = at / a.G % a.L, b = at / a.G / a.L;
  const int j = (int)(i % (2 * NP));
  if (j % NP >= a.N) return;
  const int64_t len = a.lengths ? (int64_t)a.lengths[b] : a.L;
  float v = 0.0f;
  if (l < len) {
    const float* q = a.bcpart + at * a.P * 2 * NP + j;
    for (int r = 0; r < a.P; ++r) v += q[(int64_t)r * 2 * NP];
  }
  reinterpret_cast<E*>(j < NP ? a.db : a.dc)[at * a.N + j % NP] = (E)v;
}

// dA, dD and ddelta_bias: a workgroup takes a channel's row j and adds its parts over sequences, chunks and
// group elements, each thread its own, then the threads in pairs.
template <int UNUSED = 0>
__global__ __launch_bounds__(256) void eql_scan_params_kernel(const ScanArgs a, int CH) {
  const int64_t id = a.first + blockIdx.x;
  const int ch = (int)(id / (a.N + 2)), j = (int)(id % (a.N + 2));
  float* const dst = j < a.N ? a.dA + (int64_t)ch * a.N + j : j == a.N ? (a.dD ? a.dD + ch : nullptr) : (a.dbias ? a.dbias + ch : nullptr);
  if (!dst) return;
  const int64_t n = a.B * a.K * a.T;
  float v = 0.0f;
  for (int64_t i = threadIdx.x; i < n; i += 256) {
    const int ct = ch * a.T + (int)(i % a.T), g = ct / a.CTg;
    v += a.part[(i / a.T * (a.N + 2) + j) * a.cols + g * a.nblk * CH + (ct - g * a.CTg)];
  }
  __shared__ float red[4];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) *dst = (red[0] + red[1]) + (red[2] + red[3]);
}

}  // namespace eqk
