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
// NL lanes share Q columns, two (four above 32 states), and hold four states of each in registers: a token costs a lane two
// reads of d and d x and two of b and c from LDS for 4 Q states.  Element by element work (softplus, the gate, loads and
// stores in whole vectors) runs on the tile's elements spread over all lanes; d and d x go to the
// scan through LDS, y comes back the same way.  No barrier in the forward: a wave's LDS is its own.
//
// Few columns against many tokens are split into chunks of tokens: one pass forms each chunk's state from
// zero and its sum of d, a small kernel carries the states over the chunks (a chunk multiplies what
// comes in by exp(A sum d)), and the main pass starts every chunk from its own.
//
// Bound: the vector pipe.  A state of a token costs an exponential (8 cycles of a wave) and four products or sums (4 each)
// forward, two and thirteen in the gradients; at 2.1 GHz that is 0.18 and 0.49 ps on the whole device.  Sums of four columns'
// products as fp32 MFMAs (16 x 16 x 1) gained nothing: while one runs, the SIMD issues no vector instruction.
#pragma once
#include <type_traits>

#include "eql_common.h"
#include "eql_config.h"
#include "eql_lanes.h"
#include "eql_recurrent.h"

namespace eqk {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr float kAtanh1 = 0.333333198f, kAtanh2 = 0.200038354f, kAtanh3 = 0.141169781f, kAtanh4 = 0.134337737f;

// Reads and writes of LDS by lanes of one wave stay in program order; the compiler must keep it.
__device__ __forceinline__ void wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// Q floats: one of each of a lane's columns
template <int Q>
using Cols = float __attribute__((ext_vector_type(Q)));

// Sum over the NL neighbouring lanes that share columns.
template <int NL>
__device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (NL >= 2) v += dpp<0xB1>(v);    // quad_perm 1 0 3 2
  if constexpr (NL >= 4) v += dpp<0x4E>(v);    // quad_perm 2 3 0 1
  if constexpr (NL >= 8) v += dpp<0x141>(v);   // half row mirrored: the other quad
  if constexpr (NL >= 16) v += dpp<0x140>(v);  // row mirrored: the other half
  return v;
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

// log(1 + e) / 2 for 0 <= e <= 1: atanh(s) of s = e / (2 + e) <= 1/3 is s p(s^2); p in five terms, economised from the
// series by Chebyshev polynomials over [0, 1/9], is 1.5e-8 off.
__device__ __forceinline__ float atanh_unit(float e) {
  const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
  float p = __builtin_fmaf(q, kAtanh4, kAtanh3);
  p = __builtin_fmaf(q, p, kAtanh2);
  p = __builtin_fmaf(q, p, kAtanh1);
  p = __builtin_fmaf(q, p, 1.0f);
  return s * p;
}
// NaN stays: it is one of exp(-|v|) too.
__device__ __forceinline__ float softplus(float v) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v));
  return __builtin_fmaf(2.0f, atanh_unit(e), fmaxf(v, 0.0f));
}
// softplus and its derivative from one exponential
__device__ __forceinline__ float softplus(float v, float& slope) {
  const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  slope = v < 0.0f ? e * r : r;
  return __builtin_fmaf(2.0f, atanh_unit(e), fmaxf(v, 0.0f));
}
__device__ __forceinline__ float sigmoid(float v) {  // (exp(-v) of inf gives 0)
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v));
}

// Where a wave stands; the same for all its lanes.
struct ScanPlace {
  int64_t b;       // sequence
  int k, g, blk;   // chunk, group, block of its columns
  int col0;        // first column among the padded ones
  int ct0, left;   // first column of the features, columns of the group from it on
  int64_t len;     // tokens that hold data
  int64_t begin, end;
};
template <int NL, int Q = 4>
__device__ __forceinline__ ScanPlace scan_place(const ScanArgs& a, unsigned id) {
  constexpr int CH = scan_cols(NL, Q);
  ScanPlace p;
  const unsigned nblk = Q == 4 ? a.nblk : a.bblk;
  p.blk = (int)(id % nblk);
  id /= nblk;
  p.g = (int)(id % (unsigned)a.G);
  id /= (unsigned)a.G;
  p.k = (int)(id % (unsigned)a.K);
  p.b = a.first + id / (unsigned)a.K;
  p.col0 = p.g * a.nblk * scan_cols(NL) + p.blk * CH;
  p.ct0 = p.g * a.CTg + p.blk * CH;
  p.left = a.CTg - p.blk * CH;
  p.len = a.lengths ? min(max((int64_t)a.lengths[p.b], (int64_t)0), a.L) : a.L;
  p.begin = p.k * a.chunk;
  p.end = min(p.begin + a.chunk, a.L);
  return p;
}
__device__ __forceinline__ int scan_channel(const ScanArgs& a, int ct) { return channel_of(ct, a.mT); }

constexpr uint32_t kScanDrop = 0x80000000u;  // an offset past every resource: loads give 0, stores go nowhere

// The lane's elements of a tile of [TT][CH]: NV vectors of VEC, vector v at token tok(v), column at.
// kWhole, kLoose: vectors through a buffer resource that ends behind the tile's last token, at the elements' own
// alignment.  kLoose: a group's last vector, where it is not full, is read so that it ends where the group does, and moved
// to its place as it is used (which would cost kWhole 5 %); so are the last run of a token's b and c.  kTiny (groups
// shorter than a vector, tokens further apart than 31 bits reach): single elements.
template <int DT, int NL, int MODE, int Q = 4>
struct ScanTile {
  static constexpr int CH = scan_cols(NL, Q), TT = scan_tile(NL), EPT = scan_ept(NL, Q), VEC = scan_vec(DT, NL, Q);
  static constexpr int NV = EPT / VEC, VT = CH / VEC, EB = DT == kF32 ? 4 : 2;
  static constexpr int W = VEC * EB / 4;  // 32-bit words of a vector
  static constexpr int NP = 4 * NL;
  static constexpr int NB = (TT * NL + 63) / 64;  // runs of four of b, and of c, that a lane loads
  static constexpr int BW = MODE == kLoose && NL == 1 ? 4 : EB;  // words of such a run (N < 4: one for each element)
  using E = typename Elem<DT>::T;
  struct Raw {
    uint32_t w[NV * W];
  };
  static __device__ __forceinline__ int at() { return (threadIdx.x & 63) % VT * VEC; }
  static __device__ __forceinline__ int tok(int v) { return v * (64 / VT) + (threadIdx.x & 63) / VT; }

  // whether a vector of the wave's is partly outside its group, the same for all lanes; columns of the lane's that are
  static __device__ __forceinline__ bool part(int left) { return MODE == kLoose && left < CH && left % VEC != 0; }
  static __device__ __forceinline__ int beyond(int left) { return at() < left ? max(at() + VEC - left, 0) : 0; }
  // columns before the wave's first that its resources begin with: a vector that is moved back may start there
  static __device__ __forceinline__ int lead(int left) { return part(left) ? VEC : 0; }

  // A tensor's place in the tile: the lane's byte offsets and the tokens' stride.
  struct View {
    const char* p;  // of the wave's first column, less `lead`, sequence and token 0
    int64_t stride;
    uint32_t off[MODE != kTiny ? NV : 1];
  };
  static __device__ __forceinline__ View view(const void* p, int64_t first, int64_t stride, int left) {
    View r;
    r.stride = stride;
    if constexpr (MODE != kTiny) {
      const int back = part(left) ? VEC - beyond(left) : 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) r.off[v] = at() < left ? (uint32_t)((tok(v) * (int)stride + at() + back) * EB) : kScanDrop;
    }
    return rebased(r, p, first, left);
  }
  static __device__ __forceinline__ View rebased(View r, const void* p, int64_t first, int left) {
    r.p = reinterpret_cast<const char*>(p) + (first - lead(left)) * EB;
    return r;
  }
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const View& w, int64_t l, int rows, int left) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(w.p + l * w.stride * EB), (short)0,
                                             ((rows - 1) * (int)w.stride + left + lead(left)) * EB, 0x00020000);
  }
  // tokens l .. l + nt (nt > 0); what lies behind them may be anything
  static __device__ __forceinline__ void load(Raw& r, const View& w, int64_t l, int nt, int left) {
    if constexpr (MODE != kTiny) {
      const auto rs = resource(w, l, nt, left);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if constexpr (W == 4) {
          const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, w.off[v], 0, 0));
#pragma unroll
          for (int i = 0; i < 4; ++i) r.w[v * W + i] = x[i];
        } else {
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, w.off[v], 0, 0));
          r.w[v * W] = x[0];
          r.w[v * W + 1] = x[1];
        }
      }
    } else {
      const E* p = reinterpret_cast<const E*>(w.p) + l * w.stride;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const E* q = p + tok(v) * w.stride + at();
        const int n = tok(v) < nt ? left - at() : 0;
        if constexpr (EB == 4) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) r.w[v * W + i] = i < n ? __builtin_bit_cast(uint32_t, q[i]) : 0u;
        } else {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const uint32_t lo = 2 * i < n ? h[2 * i] : 0u, hi = 2 * i + 1 < n ? h[2 * i + 1] : 0u;
            r.w[v * W + i] = lo | hi << 16;
          }
        }
      }
    }
  }
  static __device__ __forceinline__ void floats(const Raw& r, int left, float (&f)[EPT]) {
    Raw q = r;
    if (part(left)) {  // elements down by what is beyond, 0 there
      const int by = beyond(left), words = EB == 4 ? by : by / 2;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint32_t* const w = q.w + v * W;
#pragma unroll
        for (int d = 1; d < W; d *= 2)
#pragma unroll
          for (int i = 0; i < W; ++i) w[i] = words & d ? (i + d < W ? w[i + d] : 0u) : w[i];
        if constexpr (EB == 2)
#pragma unroll
          for (int i = 0; i < W; ++i) w[i] = __builtin_amdgcn_alignbit(i + 1 < W ? w[i + 1] : 0u, w[i], by % 2 * 16);
      }
    }
    // (one conversion behind the branch: with one on either side of it the compiler lost an element of the gradients' f16 tiles)
    raw_to_floats<DT, NV * W>(q.w, f);
  }
  // the same words, whose conversion is not kept from an earlier one
  static __device__ __forceinline__ void again(Raw& r) {
#pragma unroll
    for (int i = 0; i < NV * W; ++i) asm volatile("" : "+v"(r.w[i]));
  }
  static __device__ __forceinline__ void behind(float (&f)[EPT], int nt) {  // 0 from token nt on
#pragma unroll
    for (int e = 0; e < EPT; ++e) f[e] = tok(e / VEC) < nt ? f[e] : 0.0f;
  }

  // stores tokens l .. l + rows
  static __device__ __forceinline__ void store(const float (&f)[EPT], const View& w, int64_t l, int rows, int left) {
    if constexpr (MODE != kTiny) {
      const auto rs = resource(w, l, rows, left);
      const int by = part(left) ? beyond(left) : 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint32_t q[W];
#pragma unroll
        for (int i = 0; i < W; ++i) q[i] = pack2<DT>(f[v * VEC + i * (4 / EB)], f[v * VEC + i * (4 / EB) + (EB == 2)]);
        const uint32_t off = by > 0 ? kScanDrop : w.off[v];
        if constexpr (W == 4) __builtin_amdgcn_raw_buffer_store_b128(u32x4{q[0], q[1], q[2], q[3]}, rs, off, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b64(u32x2{q[0], q[1]}, rs, off, 0, 0);
        if (part(left)) {  // one element after the other
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const uint32_t o = by > 0 && i + by < VEC ? w.off[v] + (i + by) * EB : kScanDrop;
            if constexpr (EB == 4) __builtin_amdgcn_raw_buffer_store_b32(q[i], rs, o, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(q[i / 2] >> i % 2 * 16), rs, o, 0, 0);
          }
        }
      }
    } else {
      E* p = reinterpret_cast<E*>(const_cast<char*>(w.p)) + l * w.stride;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        E* q = p + tok(v) * w.stride + at();
        const int n = tok(v) < rows ? left - at() : 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (i < n) q[i] = (E)f[v * VEC + i];
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
  // b or c of a tile: runs of four, i * 64 + lane of [TT][NP / 4]
  struct Bc {
    uint32_t w[NB * BW];
  };
  static __device__ __forceinline__ void load_bc(Bc& r, const void* base, int64_t first, int64_t stride, int nt, int N) {
    const char* p = reinterpret_cast<const char*>(base) + first * EB;
    if constexpr (MODE != kTiny) {
      const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, ((nt - 1) * (int)stride + N) * EB, 0x00020000);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int j = i * 64 + (threadIdx.x & 63), t = j / NL, n = j % NL * 4;
        const bool on = n < N && t < nt;
        if (MODE == kLoose && NL == 1 && N < 4) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t off = on && q < N ? (uint32_t)((t * (int)stride + q) * EB) : kScanDrop;
            if constexpr (EB == 4) r.w[i * BW + q] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0);
            else r.w[i * BW + q] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, off, 0, 0);
          }
          continue;
        }
        // (a last run that is not full ends where the row does)
        const uint32_t off = on ? (uint32_t)((t * (int)stride + (MODE == kLoose ? min(n, N - 4) : n)) * EB) : kScanDrop;
        if constexpr (EB == 4) {
          const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
#pragma unroll
          for (int q = 0; q < 4; ++q) r.w[i * BW + q] = x[q];
        } else {
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0));
          r.w[i * BW] = x[0];
          r.w[i * BW + 1] = x[1];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int j = i * 64 + (threadIdx.x & 63), t = j / NL, n = j % NL * 4;
        const E* q = reinterpret_cast<const E*>(p) + t * stride + n;
        const int m = t < nt ? N - n : 0;
        if constexpr (EB == 4) {
#pragma unroll
          for (int o = 0; o < 4; ++o) r.w[i * BW + o] = o < m ? __builtin_bit_cast(uint32_t, q[o]) : 0u;
        } else {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
#pragma unroll
          for (int o = 0; o < 2; ++o) {
            const uint32_t lo = 2 * o < m ? h[2 * o] : 0u, hi = 2 * o + 1 < m ? h[2 * o + 1] : 0u;
            r.w[i * BW + o] = lo | hi << 16;
          }
        }
      }
    }
  }
  static __device__ __forceinline__ void put_bc(float* tile, const Bc& r, int N) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int j = i * 64 + (threadIdx.x & 63), n = j % NL * 4;
      uint32_t w[EB];
#pragma unroll
      for (int q = 0; q < EB; ++q) w[q] = r.w[i * BW + q];
      if (MODE == kLoose && NL == 1 && N < 4) {
        if constexpr (EB == 2 && BW == 4) {
          w[0] = r.w[i * BW] | r.w[i * BW + 1] << 16;
          w[1] = r.w[i * BW + 2];
        }
      } else if (MODE == kLoose && N % 4 != 0) {  // the last run's states down to their places, 0 behind them
        const int by = n < N ? max(n + 4 - N, 0) : 0;
        if constexpr (EB == 4) {
#pragma unroll
          for (int d = 1; d < 4; d *= 2)
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = by & d ? (q + d < 4 ? w[q + d] : 0u) : w[q];
        } else {
          const uint32_t lo = by & 2 ? w[1] : w[0], hi = by & 2 ? 0u : w[1];
          w[0] = __builtin_amdgcn_alignbit(hi, lo, by % 2 * 16);
          w[1] = hi >> by % 2 * 16;
        }
      }
      float f[4];
      raw_to_floats<DT, EB>(w, f);
      if (TT * NL >= 64 || j < TT * NL) *reinterpret_cast<floatx4*>(tile + j * 4) = floatx4{f[0], f[1], f[2], f[3]};
    }
  }
};

// A of states and columns that do not exist: their decay is 1 for every finite step, and 0, not NaN, for an infinite one.
constexpr float kNoDecay = -0x1p-126f;
// A of the lane's columns and four states, times log2(e); kNoDecay outside, where a state stays 0.  kWhole: four states are all
// inside or all outside, and rows of A whole 16-byte words (what lies outside is read from A's start instead).
template <int NL, int MODE, int Q>
__device__ __forceinline__ void scan_decay(const ScanArgs& a, const ScanPlace& p, float (&A2)[Q][4]) {
  const int lane = threadIdx.x & 63, n0 = lane % NL * 4, c0 = lane / NL * Q;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int m = c0 + q < p.left ? a.N - n0 : 0;
    const float* s = a.A + (m > 0 ? scan_channel(a, p.ct0 + c0 + q) * a.N + n0 : 0);
    if constexpr (MODE == kWhole) {
      const floatx4 v = *reinterpret_cast<const floatx4*>(s);
#pragma unroll
      for (int n = 0; n < 4; ++n) A2[q][n] = m > 0 ? v[n] * kLog2e : kNoDecay;
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float v = s[n < m ? n : 0];
        A2[q][n] = n < m ? v * kLog2e : kNoDecay;
      }
    }
  }
}
// The lane's states in [cols][NP] or, for the caller, [CT][N].
template <int NL, int Q>
__device__ __forceinline__ void load_padded(const float* base, float (&h)[Q][4]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(base + (lane / NL * Q + q) * (4 * NL) + lane % NL * 4);
#pragma unroll
    for (int n = 0; n < 4; ++n) h[q][n] = v[n];
  }
}
template <int NL, int Q>
__device__ __forceinline__ void store_padded(float* base, const float (&h)[Q][4]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < Q; ++q)
    *reinterpret_cast<floatx4*>(base + (lane / NL * Q + q) * (4 * NL) + lane % NL * 4) =
        floatx4{h[q][0], h[q][1], h[q][2], h[q][3]};
}
template <int NL, int Q>
__device__ __forceinline__ void load_state(const ScanArgs& a, const ScanPlace& p, const float* base, float (&h)[Q][4]) {
  const int lane = threadIdx.x & 63, n0 = lane % NL * 4, c0 = lane / NL * Q;
  const bool whole = a.N % 4 == 0 && ((uintptr_t)base & 15) == 0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const float* s = base + (p.b * a.CT + p.ct0 + c0 + q) * a.N + n0;
    if (whole) {
      const bool on = c0 + q < p.left && n0 < a.N;
      const floatx4 v = *reinterpret_cast<const floatx4*>(on ? s : base);
#pragma unroll
      for (int n = 0; n < 4; ++n) h[q][n] = on ? v[n] : 0.0f;
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const bool on = c0 + q < p.left && n0 + n < a.N;
        const float v = *(on ? s + n : base);
        h[q][n] = on ? v : 0.0f;
      }
    }
  }
}
template <int NL, int Q>
__device__ __forceinline__ void store_state(const ScanArgs& a, const ScanPlace& p, float* base, const float (&h)[Q][4]) {
  const int lane = threadIdx.x & 63, n0 = lane % NL * 4, c0 = lane / NL * Q;
  const bool whole = a.N % 4 == 0 && ((uintptr_t)base & 15) == 0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (c0 + q >= p.left || n0 >= a.N) continue;
    float* s = base + (p.b * a.CT + p.ct0 + c0 + q) * a.N + n0;
    if (whole) {
      *reinterpret_cast<floatx4*>(s) = floatx4{h[q][0], h[q][1], h[q][2], h[q][3]};
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n0 + n < a.N) s[n] = h[q][n];
    }
  }
}
// The parameter of the channels of the lane's vector, 0 outside and where src is NULL.
template <int VEC, int MODE>
__device__ __forceinline__ void scan_param(const ScanArgs& a, const ScanPlace& p, const float* src, int at, float (&f)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) f[i] = 0.0f;
  if (!src) return;
  if (MODE == kWhole && a.T % VEC == 0) {  // one channel
    const float v = src[at < p.left ? scan_channel(a, p.ct0 + at) : 0];
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = at < p.left ? v : 0.0f;
    return;
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const float v = src[at + i < p.left ? scan_channel(a, p.ct0 + at + i) : 0];
    f[i] = at + i < p.left ? v : 0.0f;
  }
}

// States past N have b = c = 0 and stay 0 as long as d x is finite: 0 times infinity is NaN, and with c = 0 that would reach
// y.  Tiles with an infinite or NaN d x are walked with those states set to 0 after each token.  In the gradients such states,
// and the columns past a group's, turn infinities to NaN only in sums that are infinite anyway.
template <int EPT>
__device__ __forceinline__ bool scan_wild(const float (&u)[EPT]) {
  float v = 0.0f;
#pragma unroll
  for (int e = 0; e < EPT; ++e) v = __builtin_fmaf(u[e], 0.0f, v);
  return __builtin_amdgcn_ballot_w64(v != v) != 0;
}

// The decays of a token: exp(d A).
template <int Q>
__device__ __forceinline__ void scan_exp(float (&e)[Q][4], const float (&A2)[Q][4], const Cols<Q>& d) {
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) e[q][n] = __builtin_amdgcn_exp2f(d[q] * A2[q][n]);
}
template <int Q>
__device__ __forceinline__ void scan_step(float (&h)[Q][4], const float (&e)[Q][4], const Cols<Q>& dx, const floatx4& bb) {
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) h[q][n] = __builtin_fmaf(e[q][n], h[q][n], dx[q] * bb[n]);
}
// End of a token in the loops over them: the next one's decays and words from LDS are on their way by then, so that one
// wave on a SIMD waits for neither (left to itself the compiler uses an exponential two instructions
// after it is issued: 980 cycles a token of 64 columns, 16 states, instead of 780).
__device__ __forceinline__ void token_end() { __builtin_amdgcn_sched_barrier(0); }

// ---- forward ---------------------------------------------------------------
// STATES: only the state that a chunk forms from zero and its sum of d (chunks 0 .. K - 2).
// Measured, f16, 16 states: 16,389 tokens of 768 columns in 114 chunks 46 us + 8 for the carry + 64; 64 x 197 tokens
// without chunks, states kept for the gradients, 62 to 67 us (0.41 ps a state of a token).  A token takes 0.19 us with one wave
// on a SIMD, 0.30 with two and 0.55 with four (with four columns a lane, for twice the work, 0.36 and 0.60, and no more fit).
template <int NL>
constexpr int scan_fwd_lds() {  // floats of a wave
  return 2 * scan_tile(NL) * scan_cols(NL, scan_columns(NL)) + 2 * scan_tile(NL) * 4 * NL;
}
template <int DT, int NL, int MODE, bool STATES>
__global__ __launch_bounds__(64 * kScanWaves, 2) void eql_scan_fwd_kernel(const ScanArgs a) {
  constexpr int Q = scan_columns(NL);
  using TL = ScanTile<DT, NL, MODE, Q>;
  using Col = Cols<Q>;
  constexpr int TT = TL::TT, CH = TL::CH, EPT = TL::EPT, VEC = TL::VEC, NP = TL::NP;
  constexpr int RUN = scan_run(NL);
  __shared__ __attribute__((aligned(16))) float lds[kScanWaves * scan_fwd_lds<NL>()];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned id = blockIdx.x * kScanWaves + wave;
  if (id >= a.tasks) return;  // (no barrier follows)
  const ScanPlace p = scan_place<NL, Q>(a, id);
  if (STATES && p.k == a.K - 1) return;
  float* const ds = lds + wave * scan_fwd_lds<NL>();
  float* const us = ds + TT * CH;
  float* const bs = us + TT * CH;
  float* const cs = bs + TT * NP;
  const int n0 = lane % NL * 4, c0 = lane / NL * Q, at = TL::at();
  const int64_t stop = min(p.len, p.end);
  const auto xv = TL::view(a.x, p.b * a.xs[0] + p.ct0, a.xs[1], p.left), dv = TL::view(a.delta, p.b * a.ds[0] + p.ct0, a.ds[1], p.left);
  const auto zv = TL::view(a.z, p.b * a.zs[0] + p.ct0, a.zs[1], p.left), yv = TL::view(a.y, p.b * a.L * a.CT + p.ct0, a.CT, p.left);
  typename TL::Raw xr, dr, zr;
  typename TL::Bc br, cr;
  auto fetch = [&](int64_t l0) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    TL::load(dr, dv, l0, nt, p.left);
    TL::load(xr, xv, l0, nt, p.left);
    TL::load_bc(br, a.b, p.b * a.bs[0] + l0 * a.bs[1] + p.g * a.bs[2], a.bs[1], nt, a.N);
    if constexpr (!STATES) {
      TL::load_bc(cr, a.c, p.b * a.cs[0] + l0 * a.cs[1] + p.g * a.cs[2], a.cs[1], nt, a.N);
      if (a.z) TL::load(zr, zv, l0, nt, p.left);
    }
  };
  if (p.begin < stop) fetch(p.begin);
  float A2[Q][4], h[Q][4], bias[VEC], skip[VEC], total[Q] = {};
  scan_decay<NL, MODE>(a, p, A2);
  scan_param<VEC, MODE>(a, p, a.bias, at, bias);
  if constexpr (!STATES) scan_param<VEC, MODE>(a, p, a.D, at, skip);
  const int64_t slot = (p.b * a.K + p.k) * a.cols + p.col0;
  if (!STATES && a.K > 1) load_padded<NL>(a.carry + slot * NP, h);
  else if (!STATES && a.h0) load_state<NL>(a, p, a.h0, h);
  else
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int n = 0; n < 4; ++n) h[q][n] = 0.0f;
  for (int64_t l0 = p.begin; l0 < stop; l0 += TT) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    typename TL::Raw xc = xr, zc = zr;  // of this tile, while the next one's are on their way
    bool wild = false;
    {
      float xf[EPT], df[EPT];
      TL::floats(dr, p.left, df);
      TL::floats(xr, p.left, xf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) df[e] += bias[e % VEC];
      if (a.softplus)
#pragma unroll
        for (int e = 0; e < EPT; ++e) df[e] = softplus(df[e]);
      if (nt < TT) {
        TL::behind(df, nt);
        TL::behind(xf, nt);
      }
      wave_order();  // the tile before has been read
      TL::put(ds, df);
#pragma unroll
      for (int e = 0; e < EPT; ++e) df[e] *= xf[e];
      TL::put(us, df);
      if (!STATES && a.N < NP) wild = scan_wild(df);  // (of a chunk's own states the carry drops those past N)
      TL::put_bc(bs, br, a.N);
      if constexpr (!STATES) TL::put_bc(cs, cr, a.N);
    }
    if (l0 + TT < stop) fetch(l0 + TT);
    if constexpr (!STATES)
      if (a.states) store_padded<NL>(a.states + ((p.b * a.runs + l0 / RUN) * a.cols + p.col0) * NP, h);
    wave_order();
    auto cols = [&](const float* tile, int t) { return *reinterpret_cast<const Col*>(tile + min(t, TT - 1) * CH + c0); };
    auto rows = [&](const float* tile, int t) { return *reinterpret_cast<const floatx4*>(tile + min(t, TT - 1) * NP + n0); };
    float part[Q] = {}, e0[Q][4], e1[Q][4];
    // y of a token, in place of its d x, which every lane of these columns has read; all of them write what all of them hold
    // (a branch here would keep the next token's reads behind it)
    auto output = [&](int t, const floatx4& cc) {
      Col y;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        float s = h[q][0] * cc[0];
#pragma unroll
        for (int n = 1; n < 4; ++n) s = __builtin_fmaf(h[q][n], cc[n], s);
        y[q] = lanes_sum<NL>(s);
      }
      *reinterpret_cast<Col*>(us + t * CH + c0) = y;
    };
    if (STATES || (nt == TT && !wild)) {
      Col d = cols(ds, 0), u = cols(us, 0);
      floatx4 bb = rows(bs, 0), cc = {};
      if constexpr (!STATES) cc = rows(cs, 0);
      scan_exp(e0, A2, d);
      Col d1 = cols(ds, 1);
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if constexpr (!STATES)
          if (t > 0 && t % RUN == 0 && a.states)
            store_padded<NL>(a.states + ((p.b * a.runs + (l0 + t) / RUN) * a.cols + p.col0) * NP, h);
        const Col d2 = cols(ds, t + 2), u1 = cols(us, t + 1);
        const floatx4 b1 = rows(bs, t + 1);
        floatx4 c1 = {};
        if constexpr (!STATES) c1 = rows(cs, t + 1);
        if (t + 1 < TT) scan_exp(e1, A2, d1);
        scan_step(h, e0, u, bb);
        if constexpr (STATES) {
#pragma unroll
          for (int q = 0; q < Q; ++q) part[q] += d[q];
        } else {
          output(t, cc);
        }
        d = d1;
        d1 = d2;
        u = u1;
        bb = b1;
        cc = c1;
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int n = 0; n < 4; ++n) e0[q][n] = e1[q][n];
        token_end();
      }
    } else {  // a sequence's last tokens, a call over few, infinities
#pragma unroll 1
      for (int t = 0; t < nt; ++t) {
        if constexpr (!STATES)
          if (t > 0 && t % RUN == 0 && a.states)
            store_padded<NL>(a.states + ((p.b * a.runs + (l0 + t) / RUN) * a.cols + p.col0) * NP, h);
        scan_exp(e0, A2, cols(ds, t));
        scan_step(h, e0, cols(us, t), rows(bs, t));
        if (wild)
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int n = 0; n < 4; ++n) h[q][n] = n0 + n < a.N ? h[q][n] : 0.0f;
        output(t, rows(cs, t));
      }
    }
    if constexpr (STATES) {
#pragma unroll
      for (int q = 0; q < Q; ++q) total[q] += part[q];
    } else {
      wave_order();
      float xf[EPT], yf[EPT];
      TL::get(us, yf);
      TL::again(xc);
      TL::floats(xc, p.left, xf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) yf[e] = __builtin_fmaf(skip[e % VEC], xf[e], yf[e]);
      if (a.z) {
        TL::again(zc);
        TL::floats(zc, p.left, xf);
#pragma unroll
        for (int e = 0; e < EPT; ++e) yf[e] *= xf[e] * sigmoid(xf[e]);
      }
      if (nt < TT) TL::behind(yf, nt);
      TL::store(yf, yv, l0, (int)min(p.end - l0, (int64_t)TT), p.left);
    }
  }
  if constexpr (STATES) {
    store_padded<NL>(a.carry + slot * NP, h);
    if (lane % NL == 0)
#pragma unroll
      for (int q = 0; q < Q; ++q) a.sums[slot + c0 + q] = total[q];
  } else {
    float zero[EPT];
#pragma unroll
    for (int e = 0; e < EPT; ++e) zero[e] = 0.0f;
    const int64_t from = p.begin + (max(stop - p.begin, (int64_t)0) + TT - 1) / TT * TT;  // tiles of padding alone
    for (int64_t l0 = from; l0 < p.end; l0 += TT) TL::store(zero, yv, l0, (int)min(p.end - l0, (int64_t)TT), p.left);
    if (a.hT && p.k == a.K - 1) store_state<NL>(a, p, a.hT, h);
  }
}

// A call over few tokens, without kept states: a wave takes its columns one token at a time, and a lane's four columns lie
// 64 / NL apart, so that states come and go in whole cache lines.  Bound by them: 256 sequences of 2048 columns of 64 f32
// states take one token in 56 us, 4.8 TB/s; the kernel of tiles, whose registers leave two waves a SIMD, in 95.  Few waves wait
// for their loads one after the other: one token of 32 sequences of 768 columns of 16 states, 5.3 us, with tiles 6.7.  From
// 6 tokens on (3 where a lane has all of a column's states) the tiles are faster there: 8 tokens 10.2 us, with tiles 8.8.
constexpr int scan_few(int NL) { return NL == 1 ? 2 : 4; }  // tokens
template <int DT, int NL>
__global__ __launch_bounds__(64 * kScanWaves) void eql_scan_few_kernel(const ScanArgs a) {
  using E = typename Elem<DT>::T;
  constexpr int CH = scan_cols(NL), NP = 4 * NL, STEP = 64 / NL, EC = CH >= 64 ? CH / 64 : 1;
  __shared__ __attribute__((aligned(16))) float lds[kScanWaves][2 * CH + 2 * NP];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned id = blockIdx.x * kScanWaves + wave;
  if (id >= a.tasks) return;  // (no barrier follows)
  const ScanPlace p = scan_place<NL>(a, id);
  const int n0 = lane % NL * 4, c0 = lane / NL, cols = min(p.left, CH);
  const bool quads = a.N % 4 == 0 && ((uintptr_t)a.h0 & 15) == 0 && ((uintptr_t)a.hT & 15) == 0 && ((uintptr_t)a.A & 15) == 0;
  // four states of column c0 + q STEP, none where m <= 0
  auto states = [&](const float* base, int64_t at, int m, float (&f)[4]) {
    if (quads) {
      const floatx4 v = *reinterpret_cast<const floatx4*>(base + (m > 0 ? at : 0));
#pragma unroll
      for (int n = 0; n < 4; ++n) f[n] = m > 0 ? v[n] : 0.0f;
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const float v = base[n < m ? at + n : 0];
        f[n] = n < m ? v : 0.0f;
      }
    }
  };
  float h[4][4], A2[4][4];
  const int64_t row = (p.b * a.CT + p.ct0) * a.N;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = c0 + q * STEP, m = c < cols ? a.N - n0 : 0;
#pragma unroll
    for (int n = 0; n < 4; ++n) h[q][n] = 0.0f;
    if (a.h0) states(a.h0, row + c * a.N + n0, m, h[q]);
    states(a.A, (int64_t)(m > 0 ? scan_channel(a, p.ct0 + c) : 0) * a.N + n0, m, A2[q]);
  }
  // the elements of a token: column lane + 64 i, and b and c of state `lane`
  float xn[EC], dn[EC], zn[EC], bn = 0.0f, cn = 0.0f, bias[EC], skip[EC];
  auto fetch = [&](int64_t l) {
    auto at = [&](const void* t, const int64_t* st, int64_t i) { return (float)reinterpret_cast<const E*>(t)[p.b * st[0] + l * st[1] + i]; };
#pragma unroll
    for (int i = 0; i < EC; ++i) {
      const int c = p.ct0 + (lane + 64 * i < cols ? lane + 64 * i : 0);
      xn[i] = at(a.x, a.xs, c);
      dn[i] = at(a.delta, a.ds, c);
      zn[i] = a.z ? at(a.z, a.zs, c) : 0.0f;
    }
    const int n = lane < a.N ? lane : 0;
    bn = at(a.b, a.bs, p.g * a.bs[2] + n);
    cn = at(a.c, a.cs, p.g * a.cs[2] + n);
    if (lane >= a.N) bn = cn = 0.0f;
  };
  if (p.len > 0) fetch(0);
#pragma unroll
  for (int i = 0; i < EC; ++i) {
    const int ch = scan_channel(a, p.ct0 + (lane + 64 * i < cols ? lane + 64 * i : 0));
    bias[i] = a.bias ? a.bias[ch] : 0.0f;
    skip[i] = a.D ? a.D[ch] : 0.0f;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) A2[q][n] *= kLog2e;
  float* const ds = lds[wave];
  float* const us = ds + CH;
  float* const bs = us + CH;
  float* const cs = bs + NP;
  E* const y = reinterpret_cast<E*>(a.y) + p.b * a.L * a.CT + p.ct0;
  for (int64_t l = 0; l < a.L; ++l) {
    float f[EC], x[EC], z[EC];
    if (l < p.len) {
#pragma unroll
      for (int i = 0; i < EC; ++i) {
        x[i] = xn[i];
        z[i] = zn[i];
        float d = dn[i] + bias[i];
        if (a.softplus) d = softplus(d);
        if (lane + 64 * i < CH) {
          ds[lane + 64 * i] = d;
          us[lane + 64 * i] = d * x[i];
        }
      }
      if (lane < NP) {
        bs[lane] = bn;
        cs[lane] = cn;
      }
      if (l + 1 < p.len) fetch(l + 1);
      wave_order();
      const floatx4 bb = *reinterpret_cast<const floatx4*>(bs + n0), cc = *reinterpret_cast<const floatx4*>(cs + n0);
      float out[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float d = ds[c0 + q * STEP], u = us[c0 + q * STEP];
        float s = 0.0f;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const float next = __builtin_fmaf(__builtin_amdgcn_exp2f(d * A2[q][n]), h[q][n], u * bb[n]);
          h[q][n] = n0 + n < a.N ? next : 0.0f;  // (0 times an infinite u)
          s = __builtin_fmaf(h[q][n], cc[n], s);
        }
        out[q] = lanes_sum<NL>(s);
      }
      wave_order();
#pragma unroll
      for (int q = 0; q < 4; ++q) us[c0 + q * STEP] = out[q];  // (lanes of a column hold the same sum)
      wave_order();
#pragma unroll
      for (int i = 0; i < EC; ++i) {
        f[i] = __builtin_fmaf(skip[i], x[i], lane + 64 * i < CH ? us[lane + 64 * i] : 0.0f);
        if (a.z) f[i] *= z[i] * sigmoid(z[i]);
      }
      wave_order();
    } else {
#pragma unroll
      for (int i = 0; i < EC; ++i) f[i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < EC; ++i)
      if (lane + 64 * i < cols) y[l * a.CT + lane + 64 * i] = (E)f[i];
  }
  if (!a.hT) return;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = c0 + q * STEP, m = c < cols ? a.N - n0 : 0;
    float* const s = a.hT + row + c * a.N + n0;
    if (quads) {
      if (m > 0) *reinterpret_cast<floatx4*>(s) = floatx4{h[q][0], h[q][1], h[q][2], h[q][3]};
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (n < m) s[n] = h[q][n];
    }
  }
}

// 2^e h + v for any finite e whose product with h is in range, 0 and infinite h too: beyond 2^126 either way the whole part of e
// goes to h's exponent.
__device__ __forceinline__ float carried(float e, float h, float v) {
  const float m = __builtin_fabsf(e);
  const float w = m <= 126.0f || m == __builtin_inff() ? 0.0f : __builtin_floorf(fminf(fmaxf(e, -1000.0f), 1000.0f));
  return __builtin_fmaf(__builtin_amdgcn_exp2f(w == 0.0f ? e : fminf(fmaxf(e - w, 0.0f), 1.0f)), __builtin_ldexpf(h, (int)w), v);
}

// Carries the states over the chunks of a sequence, in place: what a chunk formed from zero becomes what it
// starts from.  BACK: from the last chunk to the first, the gradient behind a chunk.  A thread takes one
// column's state and reads kScanAhead chunks before it needs the first.  Bound by the way through memory, once for so many
// chunks: 147 chunks of 12,288 states 9 us (one chunk ahead 27).
constexpr int kScanAhead = 32;
template <bool BACK>
__global__ __launch_bounds__(64) void eql_scan_carry_kernel(const ScanArgs a, int NP) {
  const unsigned per = (unsigned)a.cols * NP, i = blockIdx.x * 64 + threadIdx.x;
  const int64_t b = a.first + i / per;
  const int col = (int)(i % per / NP), n = (int)(i % NP);
  const int CH = 1024 / NP;  // columns of a wave's block
  const int g = col / (a.nblk * CH), in = col - g * a.nblk * CH;
  const bool real = in < a.CTg && n < a.N;
  const int ct = g * a.CTg + in;
  const float* first = BACK ? a.dhT : a.h0;
  const int64_t cstep = (BACK ? -1 : 1) * (int64_t)a.cols * NP, sstep = (BACK ? -1 : 1) * (int64_t)a.cols;
  const int from = BACK ? a.K - 1 : 0;
  float* c = a.carry + ((b * a.K + from) * a.cols + col) * NP + n;
  const float* s = a.sums + (b * a.K + from) * a.cols + col;
  const float A2 = real ? a.A[(int64_t)scan_channel(a, ct) * a.N + n] * kLog2e : 0.0f;
  float h = first && real ? first[(b * a.CT + ct) * a.N + n] : 0.0f;
  // the first chunk of the way has nothing before it; the last one's own result is not wanted; what a chunk formed of
  // states and columns that do not exist may be NaN and ends here (ALL: the wave has none of them)
  auto chunks = [&](auto count, auto all) {
    constexpr int n = decltype(count)::value;
    constexpr bool ALL = decltype(all)::value;
    const float start = h;
    float v[n], e[n], d[n];
#pragma unroll
    for (int k = 0; k < n; ++k) {
      v[k] = c[k * cstep];
      e[k] = s[k * sstep];
    }
#pragma unroll
    for (int k = 0; k < n; ++k) {
      e[k] *= A2;
      d[k] = __builtin_amdgcn_exp2f(e[k]);
    }
#pragma unroll
    for (int k = 0; k < n; ++k) {
      c[k * cstep] = ALL || real ? h : 0.0f;
      h = __builtin_fmaf(d[k], h, v[k]);
    }
    // Token by token a state may stay 0, finite or infinite where a chunk's decay is infinite or 0, and their product would be
    // NaN or infinite: those chunks again, with the decay in two factors
    if (__builtin_amdgcn_ballot_w64(real && !(__builtin_fabsf(h) < __builtin_inff())) != 0) {
      h = start;
#pragma unroll
      for (int k = 0; k < n; ++k) {
        c[k * cstep] = ALL || real ? h : 0.0f;
        h = carried(e[k], h, v[k]);
      }
    }
    c += n * cstep;
    s += n * sstep;
  };
  auto walk = [&](auto all) {
    int left = a.K - 1;
    for (; left >= kScanAhead; left -= kScanAhead) chunks(std::integral_constant<int, kScanAhead>{}, all);
    for (; left >= 4; left -= 4) chunks(std::integral_constant<int, 4>{}, all);
    for (; left > 0; --left) chunks(std::integral_constant<int, 1>{}, all);
  };
  if (__builtin_amdgcn_ballot_w64(!real) == 0) walk(std::true_type{});
  else walk(std::false_type{});
  *c = real ? h : 0.0f;
}

// ---- gradients ---------------------------------------------------------------
// r behind a chunk from zero, and its sum of d (chunks 1 .. K - 1): r = a (c s + r) from the last token to the first.
template <int DT, int NL, int MODE>
__global__ __launch_bounds__(64 * kScanWaves, 2) void eql_scan_back_kernel(const ScanArgs a) {
  constexpr int Q = scan_columns(NL);
  using TL = ScanTile<DT, NL, MODE, Q>;
  using Col = Cols<Q>;
  constexpr int TT = TL::TT, CH = TL::CH, EPT = TL::EPT, VEC = TL::VEC, NP = TL::NP;
  __shared__ __attribute__((aligned(16))) float lds[kScanWaves * scan_fwd_lds<NL>()];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned id = blockIdx.x * kScanWaves + wave;
  if (id >= a.tasks) return;  // (no barrier follows)
  const ScanPlace p = scan_place<NL, Q>(a, id);
  if (p.k == 0) return;
  float* const ds = lds + wave * scan_fwd_lds<NL>();
  float* const ss = ds + TT * CH;
  float* const cs = ss + TT * CH;
  const int n0 = lane % NL * 4, c0 = lane / NL * Q, at = TL::at();
  const int64_t stop = min(p.len, p.end);
  const auto dv = TL::view(a.delta, p.b * a.ds[0] + p.ct0, a.ds[1], p.left), gv = TL::view(a.dy, p.b * a.L * a.CT + p.ct0, a.CT, p.left);
  const auto zv = TL::view(a.z, p.b * a.zs[0] + p.ct0, a.zs[1], p.left);
  typename TL::Raw yr, dr, zr;
  typename TL::Bc cr;
  auto fetch = [&](int64_t l0) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    TL::load(dr, dv, l0, nt, p.left);
    TL::load(yr, gv, l0, nt, p.left);
    if (a.z) TL::load(zr, zv, l0, nt, p.left);
    TL::load_bc(cr, a.c, p.b * a.cs[0] + l0 * a.cs[1] + p.g * a.cs[2], a.cs[1], nt, a.N);
  };
  const int64_t tiles = (max(stop - p.begin, (int64_t)0) + TT - 1) / TT;
  if (tiles > 0) fetch(p.begin + (tiles - 1) * TT);
  float A2[Q][4], r[Q][4], bias[VEC], total[Q] = {};
  scan_decay<NL, MODE>(a, p, A2);
  scan_param<VEC, MODE>(a, p, a.bias, at, bias);
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) r[q][n] = 0.0f;
  for (int64_t tile = tiles - 1; tile >= 0; --tile) {
    const int64_t l0 = p.begin + tile * TT;
    const int nt = (int)min(stop - l0, (int64_t)TT);
    {
      float sf[EPT], df[EPT];
      TL::floats(yr, p.left, sf);
      TL::floats(dr, p.left, df);
      if (a.z) {
        float zf[EPT];
        TL::floats(zr, p.left, zf);
#pragma unroll
        for (int e = 0; e < EPT; ++e) sf[e] *= zf[e] * sigmoid(zf[e]);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) df[e] += bias[e % VEC];
      if (a.softplus)
#pragma unroll
        for (int e = 0; e < EPT; ++e) df[e] = softplus(df[e]);
      if (nt < TT) {
        TL::behind(df, nt);
        TL::behind(sf, nt);
      }
      wave_order();
      TL::put(ds, df);
      TL::put(ss, sf);
      TL::put_bc(cs, cr, a.N);
    }
    if (tile > 0) fetch(l0 - TT);
    wave_order();
    auto cols = [&](const float* tile, int t) { return *reinterpret_cast<const Col*>(tile + max(t, 0) * CH + c0); };
    auto rows = [&](const float* tile, int t) { return *reinterpret_cast<const floatx4*>(tile + max(t, 0) * NP + n0); };
    float part[Q] = {}, e0[Q][4], e1[Q][4];
    Col d = cols(ds, TT - 1), s = cols(ss, TT - 1), d1 = cols(ds, TT - 2);
    floatx4 cc = rows(cs, TT - 1);
    scan_exp(e0, A2, d);
#pragma unroll
    for (int t = TT - 1; t >= 0; --t) {
      const Col d2 = cols(ds, t - 2), s1 = cols(ss, t - 1);
      const floatx4 c1 = rows(cs, t - 1);
      if (t > 0) scan_exp(e1, A2, d1);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        part[q] += d[q];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          r[q][n] = e0[q][n] * __builtin_fmaf(cc[n], s[q], r[q][n]);
          e0[q][n] = e1[q][n];
        }
      }
      d = d1;
      d1 = d2;
      s = s1;
      cc = c1;
      token_end();
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) total[q] += part[q];
  }
  const int64_t slot = (p.b * a.K + p.k) * a.cols + p.col0;
  store_padded<NL>(a.carry + slot * NP, r);
  if (lane % NL == 0)
#pragma unroll
    for (int q = 0; q < Q; ++q) a.sums[slot + c0 + q] = total[q];
}

// The gradients.  The waves of a workgroup take neighbouring column blocks of one group and chunk, so that db
// and dc are summed over them before they leave; a tile is walked from its last run of SUB tokens to the
// first: the states of a run are formed again from the one before it, which the forward kept, and held in registers.
// What a tile's elements need twice (step, slope, gate, dy silu(z)) waits in LDS beside the scan's sums.
// Two columns a lane (four above 32 states): a run's states take 64 registers, and two waves fit a SIMD.  Bound by the vector
// pipe: a wave alone takes 0.6 us a token, two 0.9 together (with four columns, for twice the work, 1.1 us, and no second
// wave fits).  What is spilled (18 to 52 registers) is used once a tile, not in the loops over tokens.
// Measured, f16, 16 states: 64 x 197 tokens of 768 columns 172 to 187 us, 1.1 to 1.2 ps a state of a token (205 with four).
template <int NL>
constexpr int scan_bwd_lds() {  // floats of a wave
  return 7 * scan_tile(NL) * scan_cols(NL, scan_columns(NL)) + 2 * scan_tile(NL) * 4 * NL;
}
template <int NL>
constexpr int scan_red_lds() {  // floats of a wave's db and dc, twice
  return 2 * 2 * scan_tile(NL) * 4 * NL;
}
template <int NL>
constexpr int scan_bwd_bytes(int waves) {
  return waves * (scan_bwd_lds<NL>() + scan_red_lds<NL>()) * 4;
}
template <int DT, int NL, int MODE>
__global__ __launch_bounds__(64 * kScanWaves, scan_columns(NL) == 4 ? 1 : 2) void eql_scan_bwd_kernel(const ScanArgs a, int waves) {
  constexpr int Q = scan_columns(NL);
  using TL = ScanTile<DT, NL, MODE, Q>;
  using Col = Cols<Q>;
  constexpr int TT = TL::TT, CH = TL::CH, EPT = TL::EPT, VEC = TL::VEC, NP = TL::NP;
  constexpr int SUB = scan_run(NL);
  using E = typename TL::E;
  extern __shared__ __attribute__((aligned(16))) float smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroup: (sequence, chunk, group, run of `waves` blocks)
  const int run = (int)(blockIdx.x % (unsigned)a.P);
  const int blocks = Q == 4 ? a.nblk : a.bblk;
  const bool on = run * waves + wave < blocks;
  ScanPlace p = scan_place<NL, Q>(a, blockIdx.x / (unsigned)a.P * (unsigned)blocks + (unsigned)min(run * waves + wave, blocks - 1));
  if (!on) p.left = 0;
  float* const ds = smem + wave * scan_bwd_lds<NL>();
  float* const us = ds + TT * CH;
  float* const ss = us + TT * CH;
  float* const as = ss + TT * CH;  // sum_n A a g h, sum_n c h, the step's slope, sigmoid(z)
  float* const hc = as + TT * CH;
  float* const ls = hc + TT * CH;
  float* const gs = ls + TT * CH;
  float* const bs = gs + TT * CH;
  float* const cs = bs + TT * NP;
  float* const red = smem + waves * scan_bwd_lds<NL>();  // [2][waves][TT][2][NP]
  const int n0 = lane % NL * 4, c0 = lane / NL * Q, at = TL::at();
  const int64_t stop = min(p.len, p.end);
  const auto xv = TL::view(a.x, p.b * a.xs[0] + p.ct0, a.xs[1], p.left), dv = TL::view(a.delta, p.b * a.ds[0] + p.ct0, a.ds[1], p.left);
  const auto zv = TL::view(a.z, p.b * a.zs[0] + p.ct0, a.zs[1], p.left);
  const auto gv = TL::view(a.dy, p.b * a.L * a.CT + p.ct0, a.CT, p.left);  // the dense tensors
  auto dense = [&](const void* q) {
    return TL::rebased(gv, q, p.b * a.L * a.CT + p.ct0, p.left);
  };
  float A2[Q][4], g[Q][4], dA[Q][4], bias[VEC], skip[VEC], dskip[VEC], dbias[VEC];
  scan_decay<NL, MODE>(a, p, A2);
  scan_param<VEC, MODE>(a, p, a.bias, at, bias);
  scan_param<VEC, MODE>(a, p, a.D, at, skip);
#pragma unroll
  for (int i = 0; i < VEC; ++i) dskip[i] = dbias[i] = 0.0f;
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int n = 0; n < 4; ++n) g[q][n] = dA[q][n] = 0.0f;
  const int64_t slot = (p.b * a.K + p.k) * a.cols + p.col0;
  if (a.K > 1 && on) load_padded<NL>(a.carry + slot * NP, g);
  else if (a.K == 1 && a.dhT) load_state<NL>(a, p, a.dhT, g);
  float* const part = a.part + (p.b * a.K + p.k) * (a.N + 2) * a.cols + p.col0;
  int odd = 0, turns = 0;
  bool flushed = false;
  auto flush = [&] {  // the lane's sums of dA, dD and ddelta_bias to memory
    if (!on) return;
    // (lanes with the same columns lie VT apart)
    auto add = [&](float* row, float (&f)[VEC]) {
      if constexpr (TL::VT <= 16) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
          const float v = columns_sum<TL::VT>(f[i], f[i + 1], f[i + 2], f[i + 3]);  // column i + row of 16 lanes
          float* const q = row + at + i + lane / 16;
          if (lane % 16 < TL::VT) *q = flushed ? *q + v : v;
        }
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float u = f[i], v = f[i];
          swap32(u, v);
          float* const q = row + at + i;
          if (lane < TL::VT) *q = flushed ? *q + (u + v) : u + v;
        }
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = 0.0f;
    };
    add(part + (int64_t)a.N * a.cols, dskip);
    add(part + (int64_t)(a.N + 1) * a.cols, dbias);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if (n0 + n >= a.N) continue;
      Col* const q = reinterpret_cast<Col*>(part + (int64_t)(n0 + n) * a.cols + c0);
      Col v;
#pragma unroll
      for (int i = 0; i < Q; ++i) v[i] = dA[i][n];
      if (flushed) v += *q;
      *q = v;
    }
    flushed = true;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int n = 0; n < 4; ++n) dA[q][n] = 0.0f;
  };
  // the tile's elements: read ahead for the scan, and again, from the caches, for what follows it
  typename TL::Raw xr, dr, zr, yr;
  typename TL::Bc br, cr;
  auto fetch = [&](int64_t l0) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    TL::load(xr, xv, l0, nt, p.left);
    TL::load(dr, dv, l0, nt, p.left);
    TL::load(yr, gv, l0, nt, p.left);
    if (a.z) TL::load(zr, zv, l0, nt, p.left);
  };
  auto fetch_bc = [&](int64_t l0) {
    const int nt = (int)min(stop - l0, (int64_t)TT);
    TL::load_bc(br, a.b, p.b * a.bs[0] + l0 * a.bs[1] + p.g * a.bs[2], a.bs[1], nt, a.N);
    TL::load_bc(cr, a.c, p.b * a.cs[0] + l0 * a.cs[1] + p.g * a.cs[2], a.cs[1], nt, a.N);
  };
  const int64_t tiles = (max(stop - p.begin, (int64_t)0) + TT - 1) / TT;
  // the state before the run of tokens from l on, the next one on the way back
  float hs[Q][4] = {};
  auto start = [&](int64_t l) {
    if (on) load_padded<NL>(a.states + ((p.b * a.runs + l / SUB) * a.cols + p.col0) * NP, hs);
  };
  if (tiles > 0) {
    fetch(p.begin + (tiles - 1) * TT);
    fetch_bc(p.begin + (tiles - 1) * TT);
    start((stop - 1) / SUB * SUB);
  }
  for (int64_t tile = tiles - 1; tile >= 0; --tile, odd ^= 1) {
    const int64_t l0 = p.begin + tile * TT;
    const int nt = (int)min(stop - l0, (int64_t)TT);
    {
      float xf[EPT], df[EPT], sf[EPT];
      TL::floats(xr, p.left, xf);
      TL::floats(dr, p.left, df);
      TL::floats(yr, p.left, sf);
      if (a.z) {
        float zf[EPT], sg[EPT];
        TL::floats(zr, p.left, zf);
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
          sg[e] = sigmoid(zf[e]);
          sf[e] *= zf[e] * sg[e];
        }
        wave_order();
        TL::put(gs, sg);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) df[e] += bias[e % VEC];
      if (a.softplus) {
        float slope[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) df[e] = softplus(df[e], slope[e]);
        wave_order();
        TL::put(ls, slope);
      }
      if (nt < TT) {
        TL::behind(df, nt);
        TL::behind(xf, nt);
        TL::behind(sf, nt);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) dskip[e % VEC] = __builtin_fmaf(sf[e], xf[e], dskip[e % VEC]);
      wave_order();
      TL::put(ds, df);
      TL::put(ss, sf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) df[e] *= xf[e];
      TL::put(us, df);
      TL::put_bc(bs, br, a.N);
      TL::put_bc(cs, cr, a.N);
    }
    if (tile > 0) fetch_bc(l0 - TT);
    wave_order();
    float* const mine = red + ((odd * waves + wave) * TT * 2) * NP;
    auto token = [&](const float* tile_, int t) { return *reinterpret_cast<const Col*>(tile_ + t * CH + c0); };
    auto states = [&](const float* tile_, int t) { return *reinterpret_cast<const floatx4*>(tile_ + t * NP + n0); };
#pragma unroll 1
    for (int s0 = (nt - 1) / SUB * SUB; s0 >= 0; s0 -= SUB) {
      float h[Q][4], H[SUB][Q][4], e0[Q][4], e1[Q][4];  // H[i]: the state before token s0 + i
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int n = 0; n < 4; ++n) h[q][n] = hs[q][n];
      if (l0 + s0 > p.begin) start(l0 + s0 - SUB);  // while this run is worked on
      scan_exp(e0, A2, token(ds, s0));
      {
        floatx4 bb = states(bs, s0);
        Col u = token(us, s0), d1 = token(ds, s0 + 1);
#pragma unroll
        for (int i = 0; i < SUB; ++i) {
          const int t1 = s0 + (i + 1 < SUB ? i + 1 : i), t2 = s0 + (i + 2 < SUB ? i + 2 : SUB - 1);
          const floatx4 b1 = states(bs, t1);
          const Col u1 = token(us, t1), d2 = token(ds, t2);
          if (i + 1 < SUB) scan_exp(e1, A2, d1);
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int n = 0; n < 4; ++n) H[i][q][n] = h[q][n];
          scan_step(h, e0, u, bb);
#pragma unroll
          for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int n = 0; n < 4; ++n) e0[q][n] = e1[q][n];
          u = u1;
          bb = b1;
          d1 = d2;
          token_end();
        }
      }
      // the way back reads the tokens and forms the exponentials again: kept, they would take as many registers
      // as the states
      asm volatile("" ::: "memory");
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int n = 0; n < 4; ++n) asm volatile("" : "+v"(A2[q][n]));
      Col d = token(ds, s0 + SUB - 1), u = token(us, s0 + SUB - 1), s = token(ss, s0 + SUB - 1), d1 = token(ds, s0 + SUB - 2);
      floatx4 bb = states(bs, s0 + SUB - 1), cc = states(cs, s0 + SUB - 1);
      scan_exp(e0, A2, d);
      Col gb = {}, ga = {}, ch = {};
      float db[4] = {}, dc[4] = {};
      // the sums over lanes of a token are taken beside the next one's products
      auto sums = [&](int t) {
        Col v;
#pragma unroll
        for (int q = 0; q < Q; ++q) v[q] = lanes_sum<NL>(gb[q]);
        // d x of this token has been read by every lane of these columns; lanes that hold the same sums write them alike,
        // without a branch
        *reinterpret_cast<Col*>(us + t * CH + c0) = v;
#pragma unroll
        for (int q = 0; q < Q; ++q) v[q] = lanes_sum<NL>(ga[q]);
        *reinterpret_cast<Col*>(as + t * CH + c0) = v;
#pragma unroll
        for (int q = 0; q < Q; ++q) v[q] = lanes_sum<NL>(ch[q]);
        *reinterpret_cast<Col*>(hc + t * CH + c0) = v;
        mine[(t * 2) * NP + n0 + lane / 16] = columns_sum<NL>(db[0], db[1], db[2], db[3]);  // state n0 + row
        mine[(t * 2 + 1) * NP + n0 + lane / 16] = columns_sum<NL>(dc[0], dc[1], dc[2], dc[3]);
      };
#pragma unroll
      for (int i = SUB - 1; i >= 0; --i) {
        const int t = s0 + i, before = i ? t - 1 : t, before2 = i > 1 ? t - 2 : s0;
        // the tokens before are read while this one is worked on
        const Col d2 = token(ds, before2), u1 = token(us, before), s1 = token(ss, before);
        const floatx4 b1 = states(bs, before), c1 = states(cs, before);
        if (i > 0) scan_exp(e1, A2, d1);
        if (i + 1 < SUB) sums(t + 1);
#pragma unroll
        for (int n = 0; n < 4; ++n) db[n] = dc[n] = 0.0f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          float sb = 0.0f, sa = 0.0f, sc = 0.0f;
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float now = i + 1 < SUB ? H[i + 1 < SUB ? i + 1 : i][q][n] : h[q][n];  // the state after token t
            g[q][n] = __builtin_fmaf(cc[n], s[q], g[q][n]);
            dc[n] = __builtin_fmaf(s[q], now, dc[n]);
            sc = __builtin_fmaf(cc[n], now, sc);
            db[n] = __builtin_fmaf(g[q][n], u[q], db[n]);
            sb = __builtin_fmaf(g[q][n], bb[n], sb);
            g[q][n] *= e0[q][n];
            const float m = g[q][n] * H[i][q][n];
            sa = __builtin_fmaf(A2[q][n], m, sa);
            dA[q][n] = __builtin_fmaf(d[q], m, dA[q][n]);
            e0[q][n] = e1[q][n];
          }
          gb[q] = sb;
          ga[q] = sa;
          ch[q] = sc;
        }
        d = d1;
        d1 = d2;
        u = u1;
        s = s1;
        bb = b1;
        cc = c1;
        token_end();
      }
      sums(s0);
    }
    wave_order();
    {
      float xf[EPT], f[EPT], o[EPT], sf[EPT];
      TL::again(xr);
      TL::floats(xr, p.left, xf);
      const int rows = (int)min(p.end - l0, (int64_t)TT);
      if (a.z && a.dz) {
        float zf[EPT], ch[EPT], sg[EPT];
        TL::again(yr);
        TL::again(zr);
        TL::floats(yr, p.left, sf);
        TL::floats(zr, p.left, zf);
        TL::get(hc, ch);
        TL::get(gs, sg);
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
          const float y0 = __builtin_fmaf(skip[e % VEC], xf[e], ch[e]);
          ch[e] = sf[e] * y0 * sg[e] * __builtin_fmaf(zf[e], 1.0f - sg[e], 1.0f);
        }
        if (nt < TT) TL::behind(ch, nt);
        TL::store(ch, dense(a.dz), l0, rows, p.left);
      }
      TL::get(us, f);  // sum_n g b
      float sa[EPT];
      TL::get(as, sa);  // sum_n A a g h, times log2(e)
#pragma unroll
      for (int e = 0; e < EPT; ++e) o[e] = __builtin_fmaf(kLn2, sa[e], xf[e] * f[e]);
      if (a.softplus) {
        TL::get(ls, sa);
#pragma unroll
        for (int e = 0; e < EPT; ++e) o[e] *= sa[e];
      }
      TL::get(ds, sa);
      TL::get(ss, sf);
#pragma unroll
      for (int e = 0; e < EPT; ++e) f[e] = __builtin_fmaf(skip[e % VEC], sf[e], sa[e] * f[e]);
      if (nt < TT) {
        TL::behind(o, nt);
        TL::behind(f, nt);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) dbias[e % VEC] += o[e];
      TL::store(o, dense(a.ddelta), l0, rows, p.left);
      TL::store(f, dense(a.dx), l0, rows, p.left);
    }
    // sums of no more than 32 tiles in registers, so that long ones lose no digits
    if (__builtin_expect(++turns == 32 || tile == 0, 0)) {
      turns = 0;
      flush();
    }
    if (tile > 0) fetch(l0 - TT);
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
      TL::store(zero, dense(a.dx), l0, rows, p.left);
      TL::store(zero, dense(a.ddelta), l0, rows, p.left);
      if (a.dz) TL::store(zero, dense(a.dz), l0, rows, p.left);
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
  if (tiles == 0 && on)
    for (int i = lane; i < (a.N + 2) * CH; i += 64) part[(int64_t)(i / CH) * a.cols + i % CH] = 0.0f;
}

// db and dc: the parts of a token's P workgroups in order.
template <int DT>
__global__ __launch_bounds__(256) void eql_scan_bc_kernel(const ScanArgs a, int NP) {
  using E = typename Elem<DT>::T;
  const int64_t i = a.first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.B * a.L * a.G * 2 * NP) return;
  const int64_t at = i / (2 * NP), token = at / a.G, b = token / a.L, l = token - b * a.L;
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
  const unsigned id = (unsigned)a.first + blockIdx.x;
  const int ch = (int)(id / (a.N + 2)), j = (int)(id % (a.N + 2));
  float* const dst = j < a.N ? a.dA + (int64_t)ch * a.N + j : j == a.N ? (a.dD ? a.dD + ch : nullptr) : (a.dbias ? a.dbias + ch : nullptr);
  if (!dst) return;
  const int64_t n = a.B * a.K;
  float v = 0.0f;
  const int ct = ch * a.T, g = ct / a.CTg, step = 256 / a.T, first = channel_of(threadIdx.x, a.mT);
  const float* const from = a.part + (int64_t)j * a.cols + g * a.nblk * CH + (ct - g * a.CTg) + (threadIdx.x - first * a.T);
  if (first < step)
    for (int64_t i = first; i < n;) {  // 64 rows, then the sums of so many, so that many rows lose no digits
      float w = 0.0f;
      for (int k = 0; k < 64 && i < n; ++k, i += step) w += from[i * (a.N + 2) * a.cols];
      v += w;
    }
  __shared__ float red[4];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) *dst = (red[0] + red[1]) + (red[2] + red[3]);
}

}  // namespace eqk
