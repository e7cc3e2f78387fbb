// eql_rotary.h -- rotary positions with several axes, for gfx950.
//
// Heads of dh channels x T group elements, the group axis fastest.  Channel pair
// c < n turns by phi = position of the pair's axis * frequency[c], the same for
// every group element, so the map commutes with the group action:
//   y_lo = x_lo cos phi - x_hi sin phi,  y_hi = x_hi cos phi + x_lo sin phi
// with (lo, hi) = (c, c + n) or, interleaved, (2c, 2c + 1); channels from 2n on pass.
#pragma once
#include "eql_common.h"
#include "eql_config.h"

namespace eqk {

constexpr int kRotaryMaxAxes = 4;
constexpr int kRotaryMaxDim = 1024;   // elements of a head
constexpr int kRotaryAngles = 2048;   // angles of a workgroup, 16 KB
constexpr int kRotaryMaxTokens = 64;  // tokens of a workgroup

struct RotaryArgs {
  const void* x;
  void* y;
  const void* positions;
  const float* freqs;
  int64_t first, tokens, L;  // first token of a launch, B * L, L
  int64_t xs[3], ys[3];      // elements: sequence, token, head
  int64_t ps[2];             // positions: sequence, token
  int N, T, n, D;
  int ends[kRotaryMaxAxes];  // first pair past each axis
  int float_pos, interleaved, copy_rest;
  float sign;                // -1: the inverse
  int TB;                    // tokens of a workgroup
};

// A workgroup takes TB tokens: first the cosine and sine of their angles, in LDS,
// then their heads, VEC elements of both members of a pair a thread (PAIRS: T = 1
// interleaved, VEC / 2 pairs side by side).  Memory bound: an angle serves every
// head and group element of its token.  The angle is formed and reduced to a turn
// in 64 bits, so a position of many thousands costs no accuracy.  4 x 6,273 tokens of
// 16 heads of 128, bf16, strided in: 43 us, 4.8 TB/s, the rate of a large copy; 64 x 197
// tokens of 24 heads of 64, fp16: 15 us, 5.2 TB/s; the tokens of one step 4 us (launch).
template <int DT, int VEC, bool PAIRS>
__global__ __launch_bounds__(256) void eql_rotary_kernel(RotaryArgs a) {
  using E = typename Elem<DT>::T;
  struct alignas(VEC * sizeof(E)) V { E e[VEC]; };
  __shared__ float2 cs[kRotaryAngles];
  __shared__ int64_t xo[kRotaryMaxTokens], yo[kRotaryMaxTokens];
  const int64_t g0 = a.first + (int64_t)blockIdx.x * a.TB;
  const int nt = (int)(a.tokens - g0 < a.TB ? a.tokens - g0 : a.TB);
  if ((int)threadIdx.x < nt) {
    const int64_t g = g0 + threadIdx.x, b = g / a.L, l = g % a.L;
    xo[threadIdx.x] = b * a.xs[0] + l * a.xs[1];
    yo[threadIdx.x] = b * a.ys[0] + l * a.ys[1];
  }
  for (int i = threadIdx.x; i < nt * a.n; i += 256) {
    const int t = i / a.n, c = i % a.n;
    const int64_t g = g0 + t, b = g / a.L, l = g % a.L;
    int ax = 0;
#pragma unroll
    for (int k = 0; k < kRotaryMaxAxes - 1; ++k) ax += c >= a.ends[k];
    const int64_t at = b * a.ps[0] + l * a.ps[1] + ax;
    const double p = a.float_pos ? (double)((const float*)a.positions)[at] : (double)((const int*)a.positions)[at];
    const double turns = p * (double)a.freqs[c] * 0.15915494309189533577;  // 1 / 2 pi
    float sn, cn;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cn);
    cs[i] = make_float2(cn, sn * a.sign);
  }
  __syncthreads();
  const int pairs = PAIRS ? 2 * a.n / VEC : a.n * a.T / VEC;  // units of a head that turn
  const int units = pairs + (a.copy_rest ? (a.D - 2 * a.n * a.T) / VEC : 0);
  const int per = a.N * units;
  for (int i = threadIdx.x; i < nt * per; i += 256) {
    const int t = i / per, h = (i - t * per) / units, w = i - t * per - h * units;
    const E* const x = (const E*)a.x + xo[t] + h * a.xs[2];
    E* const y = (E*)a.y + yo[t] + h * a.ys[2];
    if (w >= pairs) {
      const int e = 2 * a.n * a.T + (w - pairs) * VEC;
      *(V*)(y + e) = *(const V*)(x + e);
      continue;
    }
    const float2* const q = cs + t * a.n;
    if constexpr (PAIRS) {
      V v = *(const V*)(x + w * VEC);
#pragma unroll
      for (int k = 0; k < VEC / 2; ++k) {
        const float2 u = q[w * (VEC / 2) + k];
        const float lo = (float)v.e[2 * k], hi = (float)v.e[2 * k + 1];
        v.e[2 * k] = (E)(lo * u.x - hi * u.y);
        v.e[2 * k + 1] = (E)(hi * u.x + lo * u.y);
      }
      *(V*)(y + w * VEC) = v;
    } else {
      int c = w * VEC / a.T, s = w * VEC - c * a.T;
      const int lo_at = a.interleaved ? w * VEC + c * a.T : w * VEC;
      const int hi_at = lo_at + (a.interleaved ? a.T : a.n * a.T);
      V vl = *(const V*)(x + lo_at), vh = *(const V*)(x + hi_at);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float2 u = q[c];
        const float lo = (float)vl.e[k], hi = (float)vh.e[k];
        vl.e[k] = (E)(lo * u.x - hi * u.y);
        vh.e[k] = (E)(hi * u.x + lo * u.y);
        if (++s == a.T) { s = 0; ++c; }
      }
      *(V*)(y + lo_at) = vl;
      *(V*)(y + hi_at) = vh;
    }
  }
}

}  // namespace eqk
