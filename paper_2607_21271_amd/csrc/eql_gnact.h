// eql_gnact.h -- group norm with an activation over channels-last features
// x [B, S, C, T] (K = C T contiguous elements a position), for gfx950:
//   z = (x - mean) rstd w[c] + b[c],  y = act(z),
// mean and variance of a sequence's S positions, C / G channels and T group
// elements, so that the map commutes with the group action.
//
// Every pass gives a thread VEC fixed columns of the K and lets it walk the
// positions of its workgroup's chunk, so weights and statistics are registers
// and column sums need no exchange until the end.  Forward: sums of x - x0 and its
// square per chunk and group (x0 the group's first element: no cancellation
// however far the mean lies from zero), then the map, whose workgroups add the
// chunks' sums in order.  Backward: column sums of dz and dz xhat, one small kernel for
// the sums per sequence, then dx together with dw and db.
#pragma once
#include "eql_common.h"
#include "eql_config.h"

namespace eqk {

enum GnAct { kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3 };
constexpr int kGnMaxGroups = 1024;

struct GnArgs {
  const void *x, *w, *b, *dy;
  void *y, *dx, *dw, *db;
  float* stats;   // [B, G, 2] mean, rstd
  float* part;    // forward [B, P, G, 2]; backward [B, P, K, 2]
  float* sums;    // backward [B, C, 2] sums of dz xhat and dz, then [B, G, 2] means
  int64_t B, S;
  int C, T, G, K, act;
  float eps;
  int chunks, cblocks, rows;  // chunks of `rows` positions, column blocks of 256 VEC
};

// erf by Abramowitz and Stegun 7.1.26, |error| <= 1.5e-7: below half a unit of any
// 16-bit result.  Full precision takes the library function.
template <int DT>
__device__ __forceinline__ float gn_erf(float v) {
  if constexpr (DT == kF32) {
    return erff(v);
  } else {
    const float x = __builtin_fabsf(v);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
    float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
    p = __builtin_fmaf(p, t, 1.421413741f);
    p = __builtin_fmaf(p, t, -0.284496736f);
    p = __builtin_fmaf(p, t, 0.254829592f);
    const float r = 1.0f - p * t * __builtin_amdgcn_exp2f(-1.4426950408889634f * x * x);
    return __builtin_copysignf(r, v);
  }
}
template <int DT>
__device__ __forceinline__ float gn_sigmoid(float z) {
  if constexpr (DT == kF32) return 1.0f / (1.0f + expf(-z));
  else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}
template <int DT, int ACT>
__device__ __forceinline__ float gn_act(float z) {
  if constexpr (ACT == kActRelu) return z > 0.0f ? z : z < 0.0f ? 0.0f : z;  // NaN stays
  else if constexpr (ACT == kActSilu) return z * gn_sigmoid<DT>(z);
  else if constexpr (ACT == kActGelu) return 0.5f * z * (1.0f + gn_erf<DT>(z * 0.70710678118654752f));
  else return z;
}
template <int DT, int ACT>
__device__ __forceinline__ float gn_dact(float z) {
  if constexpr (ACT == kActRelu) {
    return z > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == kActSilu) {
    const float s = gn_sigmoid<DT>(z);
    return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
  } else if constexpr (ACT == kActGelu) {
    const float g = DT == kF32 ? expf(-0.5f * z * z) : __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
    return __builtin_fmaf(z * 0.39894228040143268f, g, 0.5f * (1.0f + gn_erf<DT>(z * 0.70710678118654752f)));
  } else {
    return 1.0f;
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Where a workgroup and its threads stand: threads take columns col0 .. + VEC of
// rows first, first + step, ... below last.
struct GnPlace {
  int64_t b, first, last;
  int chunk, cb, step, rr, cv, col0, cols;  // cols: columns of the block
  bool on;
};
template <int VEC>
__device__ __forceinline__ GnPlace gn_place(const GnArgs& a, uint32_t id) {
  GnPlace p;
  const int nv = a.K / VEC;
  p.cb = id % a.cblocks;
  id /= a.cblocks;
  p.chunk = id % a.chunks;
  p.b = id / a.chunks;
  const int nvb = min(nv - p.cb * 256, 256);
  p.step = 256 / nvb;
  p.rr = threadIdx.x / nvb;
  p.cv = threadIdx.x % nvb;
  p.on = p.rr < p.step;
  p.col0 = (p.cb * 256 + p.cv) * VEC;
  p.cols = nvb * VEC;
  p.first = (int64_t)p.chunk * a.rows + p.rr;
  p.last = min((int64_t)(p.chunk + 1) * a.rows, a.S);
  return p;
}

template <int DT, int VEC>
struct GnVec {
  using E = typename Elem<DT>::T;
  struct alignas(VEC * sizeof(E)) V { E e[VEC]; };
};

// ---- forward sums ----------------------------------------------------------
template <int DT, int VEC>
__global__ __launch_bounds__(256) void eql_gn_sums_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  using V = typename GnVec<DT, VEC>::V;
  __shared__ float red[2][256 * VEC];
  const GnPlace p = gn_place<VEC>(a, blockIdx.x);
  const int gw = a.K / a.G;
  const E* const xb = (const E*)a.x + p.b * a.S * a.K;
  float s1[VEC], s2[VEC], x0[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    s1[k] = s2[k] = 0.0f;
    x0[k] = p.on ? (float)xb[(p.col0 + k) / gw * gw] : 0.0f;
  }
  if (p.on) {
#pragma unroll 4
    for (int64_t r = p.first; r < p.last; r += p.step) {
      const V v = *(const V*)(xb + r * a.K + p.col0);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float d = (float)v.e[k] - x0[k];
        s1[k] += d;
        s2[k] = __builtin_fmaf(d, d, s2[k]);
      }
    }
  }
  if (p.on) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      red[0][p.rr * p.cols + p.cv * VEC + k] = s1[k];
      red[1][p.rr * p.cols + p.cv * VEC + k] = s2[k];
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, c0 = p.cb * 256 * VEC;
  float* const out = a.part + ((p.b * a.chunks + p.chunk) * a.cblocks + p.cb) * a.G * 2;
  for (int g = threadIdx.x >> 6; g < a.G; g += 4) {
    const int lo = max(g * gw, c0) - c0, hi = min((g + 1) * gw, c0 + p.cols) - c0;
    float t1 = 0.0f, t2 = 0.0f;
    const int w = hi - lo;
    for (int i = lane; i < w * p.step; i += 64) {
      const int at = i / w * p.cols + lo + i % w;
      t1 += red[0][at];
      t2 += red[1][at];
    }
    t1 = wave_sum(t1);
    t2 = wave_sum(t2);
    if (lane == 0) {
      out[2 * g] = t1;
      out[2 * g + 1] = t2;
    }
  }
}

// ---- forward map -----------------------------------------------------------
template <int DT, int VEC, int ACT>
__global__ __launch_bounds__(256) void eql_gn_map_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  using V = typename GnVec<DT, VEC>::V;
  __shared__ float2 st[kGnMaxGroups];
  const GnPlace p = gn_place<VEC>(a, blockIdx.x);
  const int gw = a.K / a.G, parts = a.chunks * a.cblocks;
  const E* const xb = (const E*)a.x + p.b * a.S * a.K;
  {
    const int lane = threadIdx.x & 63;
    const float inv = 1.0f / ((float)a.S * (float)gw);
    const float* const part = a.part + p.b * parts * a.G * 2;
    for (int g = threadIdx.x >> 6; g < a.G; g += 4) {
      float t1 = 0.0f, t2 = 0.0f;
      for (int i = lane; i < parts; i += 64) {
        t1 += part[((int64_t)i * a.G + g) * 2];
        t2 += part[((int64_t)i * a.G + g) * 2 + 1];
      }
      t1 = wave_sum(t1) * inv;
      t2 = wave_sum(t2) * inv;
      const float var = __builtin_fmaf(-t1, t1, t2);
      if (lane == 0) {
        const float mean = (float)xb[g * gw] + t1, rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + a.eps);
        st[g] = make_float2(mean, rstd);
        if (a.stats && p.chunk == 0 && p.cb == 0) {
          a.stats[(p.b * a.G + g) * 2] = mean;
          a.stats[(p.b * a.G + g) * 2 + 1] = rstd;
        }
      }
    }
  }
  __syncthreads();
  if (!p.on) return;
  float mu[VEC], m[VEC], c[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    const int col = p.col0 + k, ch = col / a.T;
    const float2 s = st[col / gw];
    mu[k] = s.x;
    m[k] = s.y * (float)((const E*)a.w)[ch];
    c[k] = (float)((const E*)a.b)[ch];
  }
  E* const yb = (E*)a.y + p.b * a.S * a.K;
#pragma unroll 2
  for (int64_t r = p.first; r < p.last; r += p.step) {
    V v = *(const V*)(xb + r * a.K + p.col0);
#pragma unroll
    for (int k = 0; k < VEC; ++k) v.e[k] = (E)gn_act<DT, ACT>(__builtin_fmaf((float)v.e[k] - mu[k], m[k], c[k]));
    *(V*)(yb + r * a.K + p.col0) = v;
  }
}

// ---- backward --------------------------------------------------------------
template <int DT, int VEC, int ACT>
__global__ __launch_bounds__(256) void eql_gn_bsums_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  using V = typename GnVec<DT, VEC>::V;
  __shared__ float red[2][256 * VEC];
  const GnPlace p = gn_place<VEC>(a, blockIdx.x);
  const int gw = a.K / a.G;
  const E* const xb = (const E*)a.x + p.b * a.S * a.K;
  const E* const gb = (const E*)a.dy + p.b * a.S * a.K;
  float s1[VEC], s2[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) s1[k] = s2[k] = 0.0f;
  if (p.on) {
    float mu[VEC], rs[VEC], w[VEC], c[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const int col = p.col0 + k, ch = col / a.T;
      const float* const s = a.stats + (p.b * a.G + col / gw) * 2;
      mu[k] = s[0];
      rs[k] = s[1];
      w[k] = (float)((const E*)a.w)[ch];
      c[k] = (float)((const E*)a.b)[ch];
    }
#pragma unroll 2
    for (int64_t r = p.first; r < p.last; r += p.step) {
      const V v = *(const V*)(xb + r * a.K + p.col0), g = *(const V*)(gb + r * a.K + p.col0);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float xh = ((float)v.e[k] - mu[k]) * rs[k];
        const float dz = (float)g.e[k] * gn_dact<DT, ACT>(__builtin_fmaf(xh, w[k], c[k]));
        s1[k] = __builtin_fmaf(dz, xh, s1[k]);
        s2[k] += dz;
      }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      red[0][p.rr * p.cols + p.cv * VEC + k] = s1[k];
      red[1][p.rr * p.cols + p.cv * VEC + k] = s2[k];
    }
  }
  __syncthreads();
  float* const out = a.part + (p.b * a.chunks + p.chunk) * a.K * 2 + (int64_t)p.cb * 256 * VEC * 2;
  for (int i = threadIdx.x; i < p.cols * 2; i += 256) {
    float t = 0.0f;
    for (int r = 0; r < p.step; ++r) t += red[i & 1][r * p.cols + (i >> 1)];
    out[i] = t;
  }
}

// Sums over the chunks and T of one sequence's channels, and from them the
// group's means of w dz and w dz xhat: one wave a group.
template <int DT>
__global__ __launch_bounds__(256) void eql_gn_bmean_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= a.B * a.G) return;
  const int64_t b = i / a.G;
  const int g = (int)(i % a.G), cg = a.C / a.G;
  const float* const part = a.part + b * a.chunks * a.K * 2;
  float m1 = 0.0f, m2 = 0.0f;
  for (int c = g * cg + lane; c < (g + 1) * cg; c += 64) {
    float t1 = 0.0f, t2 = 0.0f;
    for (int q = 0; q < a.chunks; ++q)
      for (int t = 0; t < a.T; ++t) {
        t1 += part[((int64_t)q * a.K + c * a.T + t) * 2];
        t2 += part[((int64_t)q * a.K + c * a.T + t) * 2 + 1];
      }
    a.sums[(b * a.C + c) * 2] = t1;
    a.sums[(b * a.C + c) * 2 + 1] = t2;
    const float w = (float)((const E*)a.w)[c];
    m1 = __builtin_fmaf(w, t1, m1);
    m2 = __builtin_fmaf(w, t2, m2);
  }
  m1 = wave_sum(m1);
  m2 = wave_sum(m2);
  if (lane == 0) {
    const float inv = 1.0f / ((float)a.S * (float)(a.K / a.G));
    float* const o = a.sums + a.B * a.C * 2 + i * 2;
    o[0] = m1 * inv;
    o[1] = m2 * inv;
  }
}

// dx = rstd (w dz - mean(w dz) - xhat mean(w dz xhat)); the last workgroups add
// the channels' sums over the batch: dw, db, one wave a channel.
template <int DT, int VEC, int ACT>
__global__ __launch_bounds__(256) void eql_gn_bmap_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  using V = typename GnVec<DT, VEC>::V;
  const uint32_t main = (uint32_t)(a.B * a.chunks * a.cblocks);
  if (blockIdx.x >= main) {
    const int c = (int)(blockIdx.x - main) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (c >= a.C) return;
    float t1 = 0.0f, t2 = 0.0f;
    for (int64_t b = lane; b < a.B; b += 64) {
      t1 += a.sums[(b * a.C + c) * 2];
      t2 += a.sums[(b * a.C + c) * 2 + 1];
    }
    t1 = wave_sum(t1);
    t2 = wave_sum(t2);
    if (lane == 0) {
      ((E*)a.dw)[c] = (E)t1;
      ((E*)a.db)[c] = (E)t2;
    }
    return;
  }
  const GnPlace p = gn_place<VEC>(a, blockIdx.x);
  if (!p.on) return;
  const int gw = a.K / a.G;
  const int64_t base = p.b * a.S * a.K;
  const E *const xb = (const E*)a.x + base, *const gb = (const E*)a.dy + base;
  E* const ob = (E*)a.dx + base;
  float mu[VEC], rs[VEC], w[VEC], c[VEC], m1[VEC], m2[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    const int col = p.col0 + k, ch = col / a.T;
    const int64_t gi = p.b * a.G + col / gw;
    mu[k] = a.stats[gi * 2];
    rs[k] = a.stats[gi * 2 + 1];
    m1[k] = a.sums[a.B * a.C * 2 + gi * 2];
    m2[k] = a.sums[a.B * a.C * 2 + gi * 2 + 1];
    w[k] = (float)((const E*)a.w)[ch];
    c[k] = (float)((const E*)a.b)[ch];
  }
#pragma unroll 2
  for (int64_t r = p.first; r < p.last; r += p.step) {
    V v = *(const V*)(xb + r * a.K + p.col0);
    const V g = *(const V*)(gb + r * a.K + p.col0);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float xh = ((float)v.e[k] - mu[k]) * rs[k];
      const float dz = (float)g.e[k] * gn_dact<DT, ACT>(__builtin_fmaf(xh, w[k], c[k]));
      v.e[k] = (E)(rs[k] * (__builtin_fmaf(-xh, m1[k], __builtin_fmaf(w[k], dz, -m2[k]))));
    }
    *(V*)(ob + r * a.K + p.col0) = v;
  }
}

}  // namespace eqk
