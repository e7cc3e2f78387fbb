// eql_conv.h -- short causal convolution along the tokens, forward and gradients, for gfx950.
//   u_l = bias[c] + sum_w weight[c, w] x_{l - W + 1 + w},  y = act(u)
//   du = dy act'(u);  dx_l = sum_w weight[c, w] du_{l + W - 1 - w};  dweight[c, w] = sum du_l x_{l - W + 1 + w}
// A thread takes VEC neighbouring columns (channel, group element) of a strip of tokens.  What a strip needs
// of its neighbours, W - 1 tokens, is read again, from the caches.  Runs of GR columns that share a channel share their
// weights and their sums for dweight and dbias.
// Bound: memory, and the loads that a thread has in flight: the forward reads its whole strip before it starts, the
// backward four tokens while it works on the four before (with eight at a time 36 us below, not 25: fewer waves fit).
// Measured, four taps, silu: 16,389 tokens of 768 f16 columns 16 us (3.1 TB/s), 8 x 4,096 of 1,024 28 us (4.7 TB/s);
// 25,092 tokens of 512 bf16 columns 15 us forward, 25 back (3.1 TB/s) and 5 for the parameters.
#pragma once
#include "eql_colsum.h"
#include "eql_common.h"
#include "eql_config.h"
#include "eql_recurrent.h"
#include "eql_slices.h"
#include "eql_vectors.h"

namespace eqk {

__device__ __forceinline__ float conv_sigmoid(float v) {  // (exp(-v) of inf gives 0)
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v));
}

// VEC elements as raw words.
template <int DT, int VEC>
struct ConvVec {
  static constexpr int EB = Elem<DT>::bytes, W = VEC * EB / 4;
  uint32_t w[W];
};
template <int DT, int VEC, int MODE>
__device__ __forceinline__ void conv_load(const void* p, int n, ConvVec<DT, VEC>& r) {
  load_vector<DT, VEC, MODE>(p, n, r.w);
}
template <int DT, int VEC>
__device__ __forceinline__ void conv_floats(const ConvVec<DT, VEC>& r, float (&f)[VEC]) {
  raw_to_floats<DT, ConvVec<DT, VEC>::W>(r.w, f);
}
// Where a thread stands: columns col + skip .. col + n, tokens l0 .. l1 of sequence b (none where it has no work).
struct ConvPlace {
  int64_t b, group, l0, l1, len;
  int col, skip, n, vector, turn;  // vector: among its workgroup's; turn: strip of the workgroup's
  bool has, on;                    // whether there is such a vector, and such a strip
};
template <int DT, int VEC, int MODE>
__device__ __forceinline__ void conv_store(void* p, const ConvPlace& at, const float (&f)[VEC]) {
  store_vector<DT, VEC, MODE>(p, at.skip, at.n, f);
}
template <int VEC, int MODE>
__host__ __device__ __forceinline__ ConvPlace conv_place(const ConvArgs& a, unsigned block, int thread) {
  ConvPlace p;
  const int nv = (a.CT + VEC - 1) / VEC;
  const SlicePlace at = slice_place(a.seq, a.first, block, (unsigned)(a.groups * a.cblocks));
  const int cb = (int)(at.at % (unsigned)a.cblocks);
  p.group = at.at / (unsigned)a.cblocks;
  p.b = at.seq;
  p.vector = thread % a.width;
  p.turn = thread / a.width;
  p.has = cb * a.width + p.vector < nv;
  p.col = (cb * a.width + p.vector) * VEC;
  p.skip = 0;
  p.n = MODE == kTiny ? a.CT : VEC;
  if constexpr (MODE == kLoose) {
    p.skip = p.col > a.CT - VEC ? p.col - (a.CT - VEC) : 0;
    p.col -= p.skip;
  }
  const int64_t strip = p.group * a.turns + p.turn;
  p.on = p.turn < a.turns && strip < a.strips && p.has;
  const int64_t n = a.lengths ? a.lengths[p.b] : a.L;
  p.len = n < 0 ? 0 : n > a.L ? a.L : n;
  p.l0 = p.on ? strip * a.rows : 0;
  p.l1 = !p.on ? 0 : p.l0 + a.rows < a.L ? p.l0 + a.rows : a.L;
  return p;
}
template <int DT, int W, int VEC, int GR>
__device__ __forceinline__ void conv_weights(const ConvArgs& a, const ConvPlace& p, float (&w)[W][VEC / GR], float (&bias)[VEC / GR]) {
  using E = typename Elem<DT>::T;
#pragma unroll
  for (int i = 0; i < VEC / GR; ++i) {
    const int c = channel_of(min(p.col + i * GR, a.CT - 1), a.mT);
    bias[i] = a.bias ? (float)reinterpret_cast<const E*>(a.bias)[c] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = (float)reinterpret_cast<const E*>(a.w)[c * W + j];
  }
}
// Token l of sequence b, from the state before token 0; 0 from len on, before the state, and for a thread without work.
template <int DT, int W, int VEC, int MODE>
__device__ __forceinline__ void conv_token(const ConvArgs& a, const ConvPlace& p, int64_t l, ConvVec<DT, VEC>& r) {
  constexpr int EB = Elem<DT>::bytes;
  if (p.on && l >= 0 && l < p.len) {
    conv_load<DT, VEC, MODE>((const char*)a.x + (p.b * a.xs[0] + l * a.xs[1] + p.col) * EB, p.n, r);
  } else if (p.on && l < 0 && a.h0) {
    conv_load<DT, VEC, MODE>((const char*)a.h0 + ((p.b * (W - 1) + l + W - 1) * a.CT + p.col) * EB, p.n, r);
  } else {
#pragma unroll
    for (int i = 0; i < ConvVec<DT, VEC>::W; ++i) r.w[i] = 0u;
  }
}

constexpr int kConvRows = 16;  // of a forward strip

template <int DT, int W, int VEC, int GR, int MODE>
__global__ __launch_bounds__(256) void eql_conv_fwd_kernel(const ConvArgs a) {
  constexpr int EB = Elem<DT>::bytes;
  const ConvPlace p = conv_place<VEC, MODE>(a, blockIdx.x, (int)threadIdx.x);
  if (!p.on) return;
  ConvVec<DT, VEC> raw[kConvRows + W - 1];  // tokens l0 - (W - 1) ..
  const bool inner = p.l0 >= W - 1 && p.l0 + kConvRows <= p.len;
  if (inner) {
    const char* q = (const char*)a.x + (p.b * a.xs[0] + (p.l0 - (W - 1)) * a.xs[1] + p.col) * EB;
#pragma unroll
    for (int j = 0; j < kConvRows + W - 1; ++j) conv_load<DT, VEC, MODE>(q + j * a.xs[1] * EB, p.n, raw[j]);
  } else {
#pragma unroll
    for (int j = 0; j < kConvRows + W - 1; ++j) conv_token<DT, W, VEC, MODE>(a, p, p.l0 - (W - 1) + j, raw[j]);
  }
  float w[W][VEC / GR], bias[VEC / GR], x[W][VEC];  // x[W - 1]: the newest token
  conv_weights<DT, W, VEC, GR>(a, p, w, bias);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) conv_floats(raw[j], x[j + 1]);
  char* out = (char*)a.y + ((p.b * a.L + p.l0) * a.CT + p.col) * EB;
#pragma unroll
  for (int r = 0; r < kConvRows; ++r) {
    if (p.l0 + r >= p.l1) break;
    float y[VEC];
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j][i] = x[j + 1][i];
    conv_floats(raw[r + W - 1], x[W - 1]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      y[i] = bias[i / GR];
#pragma unroll
      for (int j = 0; j < W; ++j) y[i] = __builtin_fmaf(w[j][i / GR], x[j][i], y[i]);
      if (a.silu) y[i] *= conv_sigmoid(y[i]);
    }
    if (p.l0 + r >= p.len)
#pragma unroll
      for (int i = 0; i < VEC; ++i) y[i] = 0.0f;
    conv_store<DT, VEC, MODE>(out + (int64_t)r * a.CT * EB, p, y);
  }
  // the last W - 1 tokens: the first strip alone reads the state, so it may be updated in place
  if (W > 1 && a.hT && p.l0 == 0) {
    ConvVec<DT, VEC> s[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) conv_token<DT, W, VEC, MODE>(a, p, p.len - (W - 1) + j, s[j]);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      float f[VEC];
      conv_floats(s[j], f);
      conv_store<DT, VEC, MODE>((char*)a.hT + ((p.b * (W - 1) + j) * a.CT + p.col) * EB, p, f);
    }
  }
}

// dx of the strip's tokens; its sums for dweight and dbias.  du of the W - 1 tokens behind the strip is formed again:
// rows + W - 1 tokens are walked, a multiple of eight, in batches.
constexpr int kConvBatch = 4;

template <int DT, int W, int VEC, int GR, int MODE>
__global__ __launch_bounds__(256) void eql_conv_bwd_kernel(const ConvArgs a) {
  constexpr int EB = Elem<DT>::bytes, NG = VEC / GR;
  const ConvPlace p = conv_place<VEC, MODE>(a, blockIdx.x, (int)threadIdx.x);
  const int steps = a.rows + W - 1;
  const bool inner = p.on && p.l0 >= W - 1 && p.l0 + steps <= p.len;
  ConvVec<DT, VEC> xr[kConvBatch], gr[kConvBatch], before[W];
  const char* const xp = (const char*)a.x + (p.b * a.xs[0] + p.l0 * a.xs[1] + p.col) * EB;
  const char* const gp = (const char*)a.dy + ((p.b * a.L + p.l0) * a.CT + p.col) * EB;
  auto fetch = [&](int s) {
    if (inner) {
#pragma unroll
      for (int j = 0; j < kConvBatch; ++j) {
        conv_load<DT, VEC, MODE>(xp + (int64_t)(s + j) * a.xs[1] * EB, p.n, xr[j]);
        conv_load<DT, VEC, MODE>(gp + (int64_t)(s + j) * a.CT * EB, p.n, gr[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kConvBatch; ++j) {
        conv_token<DT, W, VEC, MODE>(a, p, p.l0 + s + j, xr[j]);
        if (p.on && p.l0 + s + j < p.len) conv_load<DT, VEC, MODE>(gp + (int64_t)(s + j) * a.CT * EB, p.n, gr[j]);
        else
#pragma unroll
          for (int i = 0; i < ConvVec<DT, VEC>::W; ++i) gr[j].w[i] = 0u;
      }
    }
  };
#pragma unroll
  for (int j = 0; j < W - 1; ++j) conv_token<DT, W, VEC, MODE>(a, p, p.l0 - (W - 1) + j, before[j]);
  fetch(0);
  float w[W][NG], bias[NG], x[W][VEC], du[W][VEC], dw[W][NG], db[NG];
  conv_weights<DT, W, VEC, GR>(a, p, w, bias);
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    db[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][i] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) du[j][i] = 0.0f;
#pragma unroll
  for (int j = 0; j < W - 1; ++j) conv_floats(before[j], x[j + 1]);
  // du[j]: of token l - (W - 1) + j
  for (int s = 0; s < steps; s += kConvBatch) {
    ConvVec<DT, VEC> xc[kConvBatch], gc[kConvBatch];
#pragma unroll
    for (int j = 0; j < kConvBatch; ++j) {
      xc[j] = xr[j];
      gc[j] = gr[j];
    }
    if (s + kConvBatch < steps) fetch(s + kConvBatch);
#pragma unroll
    for (int r = 0; r < kConvBatch; ++r) {
      const int64_t l = p.l0 + s + r;
#pragma unroll
      for (int j = 0; j + 1 < W; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          x[j][i] = x[j + 1][i];
          du[j][i] = du[j + 1][i];
        }
      conv_floats(xc[r], x[W - 1]);
      float g[VEC];
      conv_floats(gc[r], g);
      if (a.silu) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float u = bias[i / GR];
#pragma unroll
          for (int j = 0; j < W; ++j) u = __builtin_fmaf(w[j][i / GR], x[j][i], u);
          const float sg = conv_sigmoid(u);
          g[i] *= sg * __builtin_fmaf(u, 1.0f - sg, 1.0f);
        }
      }
      if (!inner && l >= p.len)  // (a gradient of 0 behind the sequence, whatever the weights)
#pragma unroll
        for (int i = 0; i < VEC; ++i) g[i] = 0.0f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) du[W - 1][i] = g[i];
      if (l < p.l1) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          db[i / GR] += g[i];
#pragma unroll
          for (int j = 0; j < W; ++j) dw[j][i / GR] = __builtin_fmaf(g[i], x[j][i], dw[j][i / GR]);
        }
      }
      // token l - (W - 1) has its last du; what falls before token 0 is the state's
      const int64_t at = l - (W - 1);
      if (!p.on || at >= p.l1 || !(at >= p.l0 || (at < 0 && a.dh0))) continue;
      float d[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        d[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) d[i] = __builtin_fmaf(w[W - 1 - j][i / GR], du[j][i], d[i]);
      }
      if (!inner) {
        if (W > 1 && a.dhT && at >= p.len - (W - 1) && at < p.len) {  // a token of the last ones
          ConvVec<DT, VEC> hr;
          float h[VEC];
          conv_load<DT, VEC, MODE>((const char*)a.dhT + ((p.b * (W - 1) + at - p.len + W - 1) * a.CT + p.col) * EB, p.n, hr);
          conv_floats(hr, h);
#pragma unroll
          for (int i = 0; i < VEC; ++i) d[i] += h[i];
        }
        if (at >= p.len)
#pragma unroll
          for (int i = 0; i < VEC; ++i) d[i] = 0.0f;
      }
      if (at >= 0) conv_store<DT, VEC, MODE>((char*)a.dx + ((p.b * a.L + at) * a.CT + p.col) * EB, p, d);
      else conv_store<DT, VEC, MODE>((char*)a.dh0 + ((p.b * (W - 1) + at + W - 1) * a.CT + p.col) * EB, p, d);
    }
  }
  // the sums of the workgroup's strips, in order
  __shared__ float red[256][NG];
  const int K = a.CT / GR;
  float* const part = a.part + (p.b * a.groups + p.group) * (W + 1) * K + p.col / GR;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    if (j) __syncthreads();
#pragma unroll
    for (int i = 0; i < NG; ++i) red[threadIdx.x][i] = j < W ? dw[j < W ? j : 0][i] : db[i];
    __syncthreads();
    if (p.turn == 0 && p.has) {
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        if (i * GR < p.skip || i * GR >= p.n) continue;
        float v = red[p.vector][i];
        for (int t = 1; t < a.turns; ++t) v += red[t * a.width + p.vector][i];
        part[(int64_t)j * K + i] = v;
      }
    }
  }
}

// dweight and dbias from the workgroups' sums.
template <int DT>
__global__ __launch_bounds__(kColsumThreads) void eql_conv_params_kernel(const ConvArgs a, int GR) {
  using E = typename Elem<DT>::T;
  const int j = (int)(blockIdx.x % (a.W + 1)), block = (int)(blockIdx.x / (a.W + 1));
  const int T = a.T / GR, K = a.C * T;
  column_sums(a.part + (int64_t)j * K, a.B * a.groups, (int64_t)(a.W + 1) * K, a.C, T, block, [&](int c, float v) {
    if (j < a.W) reinterpret_cast<E*>(a.dw)[(int64_t)c * a.W + j] = (E)v;
    else if (a.db) reinterpret_cast<E*>(a.db)[c] = (E)v;
  });
}

}  // namespace eqk
