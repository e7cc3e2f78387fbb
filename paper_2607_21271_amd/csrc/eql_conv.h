// eql_conv.h -- short causal convolution along the tokens, forward and gradients, for gfx950.
//   u_l = bias[c] + sum_w weight[c, w] x_{l - W + 1 + w},  y = act(u)
//   du = dy act'(u);  dx_l = sum_w weight[c, w] du_{l + W - 1 - w};  dweight[c, w] = sum du_l x_{l - W + 1 + w}
// A thread takes VEC neighbouring columns (channel, group element) of a strip of tokens and keeps the window
// of W tokens in registers; what a strip needs of its neighbours is read again (W - 1 tokens, from the caches).
// Bound: memory.
#pragma once
#include "eql_common.h"
#include "eql_config.h"
#include "eql_recurrent.h"

namespace eqk {

template <int DT>
__device__ __forceinline__ float conv_sigmoid(float v) {
  const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * __builtin_fabsf(v));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  return v < 0.0f ? e * r : r;
}

// VEC elements at p, as floats; WHOLE: one aligned vector, else `n` single ones (the others 0).
template <int DT, int VEC, bool WHOLE>
__device__ __forceinline__ void conv_load(const void* p, int n, float (&f)[VEC]) {
  using E = typename Elem<DT>::T;
  if constexpr (WHOLE) {
    constexpr int W = VEC * Elem<DT>::bytes / 4;
    uint32_t w[W];
    if constexpr (W == 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else {
      const u32x2 v = *reinterpret_cast<const u32x2*>(p);
      w[0] = v[0];
      w[1] = v[1];
    }
    raw_to_floats<DT, W>(w, f);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = i < n ? (float)reinterpret_cast<const E*>(p)[i] : 0.0f;
  }
}
template <int DT, int VEC, bool WHOLE>
__device__ __forceinline__ void conv_store(void* p, int n, const float (&f)[VEC]) {
  using E = typename Elem<DT>::T;
  if constexpr (WHOLE) {
    constexpr int EB = Elem<DT>::bytes, W = VEC * EB / 4;
    uint32_t w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = pack2<DT>(f[i * (4 / EB)], f[i * (4 / EB) + (EB == 2)]);
    if constexpr (W == 4) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
    else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < n) reinterpret_cast<E*>(p)[i] = (E)f[i];
  }
}

// Where a thread stands: columns col .. col + n, tokens l0 .. l1 of sequence b.
struct ConvPlace {
  int64_t b, strip, l0, l1, len;
  int col, n;
};
template <int VEC>
__device__ __forceinline__ bool conv_place(const ConvArgs& a, ConvPlace& p) {
  const int nv = (a.CT + VEC - 1) / VEC;
  const int64_t i = (a.first + blockIdx.x) * 256 + threadIdx.x;
  p.col = (int)(i % nv) * VEC;
  p.n = min(VEC, a.CT - p.col);
  p.strip = i / nv % a.strips;
  p.b = i / nv / a.strips;
  if (p.b >= a.B) return false;
  p.len = a.lengths ? min(max((int64_t)a.lengths[p.b], (int64_t)0), a.L) : a.L;
  p.l0 = p.strip * a.rows;
  p.l1 = min(p.l0 + a.rows, a.L);
  return true;
}
template <int DT, int W, int VEC>
__device__ __forceinline__ void conv_weights(const ConvArgs& a, const ConvPlace& p, float (&w)[W][VEC], float (&bias)[VEC]) {
  using E = typename Elem<DT>::T;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = min(p.col + i, a.CT - 1) / a.T;
    bias[i] = a.bias ? (float)reinterpret_cast<const E*>(a.bias)[c] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = (float)reinterpret_cast<const E*>(a.w)[c * W + j];
  }
}
// Token l of sequence b, from the state before token 0; 0 from len on and before the state.
template <int DT, int W, int VEC, bool WHOLE>
__device__ __forceinline__ void conv_token(const ConvArgs& a, const ConvPlace& p, int64_t l, float (&f)[VEC]) {
  constexpr int EB = Elem<DT>::bytes;
  if (l >= 0 && l < p.len) {
    conv_load<DT, VEC, WHOLE>((const char*)a.x + (p.b * a.xs[0] + l * a.xs[1] + p.col) * EB, p.n, f);
  } else if (l < 0 && a.h0) {
    conv_load<DT, VEC, WHOLE>((const char*)a.h0 + ((p.b * (W - 1) + l + W - 1) * a.CT + p.col) * EB, p.n, f);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = 0.0f;
  }
}

template <int DT, int W, int VEC, bool WHOLE>
__global__ __launch_bounds__(256) void eql_conv_fwd_kernel(const ConvArgs a) {
  constexpr int EB = Elem<DT>::bytes;
  ConvPlace p;
  if (!conv_place<VEC>(a, p)) return;
  float w[W][VEC], bias[VEC], x[W][VEC];  // x[W - 1]: the newest token
  conv_weights<DT, W, VEC>(a, p, w, bias);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) conv_token<DT, W, VEC, WHOLE>(a, p, p.l0 - (W - 1) + j, x[j + 1]);
#pragma unroll 4
  for (int64_t l = p.l0; l < p.l1; ++l) {
    float y[VEC];
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j][i] = x[j + 1][i];
    conv_token<DT, W, VEC, WHOLE>(a, p, l, x[W - 1]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      y[i] = bias[i];
#pragma unroll
      for (int j = 0; j < W; ++j) y[i] = __builtin_fmaf(w[j][i], x[j][i], y[i]);
      if (a.silu) y[i] *= conv_sigmoid<DT>(y[i]);
      if (l >= p.len) y[i] = 0.0f;
    }
    conv_store<DT, VEC, WHOLE>((char*)a.y + ((p.b * a.L + l) * a.CT + p.col) * EB, p.n, y);
  }
  // the last W - 1 tokens: the first strip alone reads the state, so it may be updated in place
  if (W > 1 && a.hT && p.strip == 0) {
    float s[W][VEC];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) conv_token<DT, W, VEC, WHOLE>(a, p, p.len - (W - 1) + j, s[j]);
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
      conv_store<DT, VEC, WHOLE>((char*)a.hT + ((p.b * (W - 1) + j) * a.CT + p.col) * EB, p.n, s[j]);
  }
}

// dx of the strip's tokens; its sums for dweight and dbias.  du of the W - 1 tokens behind the strip is formed again.
template <int DT, int W, int VEC, bool WHOLE>
__global__ __launch_bounds__(256) void eql_conv_bwd_kernel(const ConvArgs a) {
  constexpr int EB = Elem<DT>::bytes;
  ConvPlace p;
  if (!conv_place<VEC>(a, p)) return;
  float w[W][VEC], bias[VEC], x[W][VEC], du[W][VEC], dw[W][VEC], db[VEC];
  conv_weights<DT, W, VEC>(a, p, w, bias);
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    db[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][i] = du[j][i] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j < W - 1; ++j) conv_token<DT, W, VEC, WHOLE>(a, p, p.l0 - (W - 1) + j, x[j + 1]);
  // du[j]: of token l - (W - 1) + j
#pragma unroll 2
  for (int64_t l = p.l0; l < p.l1 + W - 1; ++l) {
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        x[j][i] = x[j + 1][i];
        du[j][i] = du[j + 1][i];
      }
    conv_token<DT, W, VEC, WHOLE>(a, p, l, x[W - 1]);
    float g[VEC];
    if (l < p.len) conv_load<DT, VEC, WHOLE>((const char*)a.dy + ((p.b * a.L + l) * a.CT + p.col) * EB, p.n, g);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (l >= p.len) {
        g[i] = 0.0f;
      } else if (a.silu) {
        float u = bias[i];
#pragma unroll
        for (int j = 0; j < W; ++j) u = __builtin_fmaf(w[j][i], x[j][i], u);
        const float s = conv_sigmoid<DT>(u);
        g[i] *= s * __builtin_fmaf(u, 1.0f - s, 1.0f);
      }
      du[W - 1][i] = g[i];
      if (l < p.l1) {
        db[i] += g[i];
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][i] = __builtin_fmaf(g[i], x[j][i], dw[j][i]);
      }
    }
    // token l - (W - 1) has its last du; of the strip before, what falls before token 0 is the state's
    const int64_t at = l - (W - 1);
    const bool mine = at >= p.l0 || (at < 0 && a.dh0);
    if (mine) {
      float d[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        d[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) d[i] = __builtin_fmaf(w[W - 1 - j][i], du[j][i], d[i]);
      }
      if (W > 1 && a.dhT && at >= p.len - (W - 1) && at < p.len) {  // a token of the last ones
        float h[VEC];
        conv_load<DT, VEC, WHOLE>((const char*)a.dhT + ((p.b * (W - 1) + at - p.len + W - 1) * a.CT + p.col) * EB, p.n, h);
#pragma unroll
        for (int i = 0; i < VEC; ++i) d[i] += h[i];
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) d[i] = at < p.len ? d[i] : 0.0f;
      if (at >= 0) conv_store<DT, VEC, WHOLE>((char*)a.dx + ((p.b * a.L + at) * a.CT + p.col) * EB, p.n, d);
      else conv_store<DT, VEC, WHOLE>((char*)a.dh0 + ((p.b * (W - 1) + at + W - 1) * a.CT + p.col) * EB, p.n, d);
    }
  }
  float* const part = a.part + (p.b * a.strips + p.strip) * (W + 1) * a.CT + p.col;
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < p.n) part[(int64_t)j * a.CT + i] = j < W ? dw[j < W ? j : 0][i] : db[i];
}

// dweight and dbias: a workgroup adds the parts of one channel and weight.
template <int DT>
__global__ __launch_bounds__(256) void eql_conv_params_kernel(const ConvArgs a) {
  using E = typename Elem<DT>::T;
  const int64_t id = a.first + blockIdx.x;
  const int ch = (int)(id / (a.W + 1)), j = (int)(id % (a.W + 1));
  E* const dst = j < a.W ? reinterpret_cast<E*>(a.dw) + (int64_t)ch * a.W + j : a.db ? reinterpret_cast<E*>(a.db) + ch : nullptr;
  if (!dst) return;
  const int64_t n = a.B * a.strips * a.T;
  float v = 0.0f;
  for (int64_t i = threadIdx.x; i < n; i += 256) v += a.part[(i / a.T * (a.W + 1) + j) * a.CT + ch * a.T + i % a.T];
  __shared__ float red[4];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) *dst = (E)((red[0] + red[1]) + (red[2] + red[3]));
}

}  // namespace eqk
