// eql_resnorm.h -- the residual sum between two norms, forward and gradients, for gfx950.
//   v = norm(u) pw + pb (or u);  r = x + k v, k = scale[c] gate[b, c];  h = norm(r) w + b
// over the K = C T elements of a token, per-channel parameters shared over T.  With rh, uh the normalised rows and
// fr, fu their factors:
//   dr' = dr + fr (q - mean(q) - rh mean(q rh)), q = dh w  (rms: without mean(q));  dx = dr'
//   du = k dr', or through the norm before: fu (p - mean(p) - uh mean(p uh)), p = k dr' pw
//   dw = sum dh rh, db = sum dh;  with E = sum dr' v, P = sum dr' uh, S = sum dr' over a sequence's tokens and T:
//   E = pw P + pb S where there is a norm before, dgate = scale E, dscale = sum_b gate E, dpw = sum_b k P,
//   dpb = sum_b k S.
// LANES threads hold a row, EPT elements each, and walk the rows of their strip; means are two-pass, from
// registers.  The backward forms r again from x and u: what it reads is the inputs and the two gradients, and
// no rounding of r enters.  Column sums stay in registers over a strip, then one row of sums a workgroup goes to
// memory, and two small kernels add them in a fixed order.
// Bound: memory (forward 4, backward 6 rows an element), in the backward with the waves that its sums leave.
// Measured: 12,608 rows of 768 f16 17 us forward (4.6 TB/s), 26 back (4.5 TB/s) and 9 for the parameters; 25,092
// rows of 1,024 bf16 with a norm before and after 40 and 66 us (5.1 and 4.7 TB/s).
#pragma once
#include "eql_colsum.h"
#include "eql_common.h"
#include "eql_config.h"
#include "eql_lanes.h"
#include "eql_recurrent.h"
#include "eql_slices.h"
#include "eql_vectors.h"

namespace eqk {

template <int DT, int LANES, int EPT, int MODE, int GR>
struct ResRow {
  using E = typename Elem<DT>::T;
  static constexpr int EB = Elem<DT>::bytes, VEC = 16 / EB, NV = EPT / VEC;
  static constexpr int NP = EPT / GR;  // parameters of a thread: of runs of GR columns that share a channel
  static_assert(LANES >= 4 && (LANES & (LANES - 1)) == 0);
  static constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;   // rows of a workgroup at a time
  static constexpr int THREADS = LANES < 256 ? 256 : LANES;
  struct Raw {
    uint32_t w[NV * 4];
  };
  // first element of vector v, where it would be in a row of whole vectors and where it is
  static __device__ __forceinline__ int place(int v) { return (v * LANES + (int)(threadIdx.x % LANES)) * VEC; }
  static __device__ __forceinline__ int at(int v, int K) { return MODE == kLoose ? min(place(v), K - VEC) : place(v); }
  // whether the thread's element e is its own
  static __device__ __forceinline__ bool own(int e, int K) {
    if constexpr (MODE == kLoose) return e % VEC >= place(e / VEC) - (K - VEC);
    return place(e / VEC) + (MODE == kTiny ? e % VEC : 0) < K;
  }
  static __device__ __forceinline__ void load(Raw& r, const void* base, int64_t row, int K, bool on) {
    const E* p = reinterpret_cast<const E*>(base) + row * K;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (on && place(v) < K) {
        load_vector<DT, VEC, MODE>(p + at(v, K), K, r.w + v * 4);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[v * 4 + i] = 0u;
      }
    }
  }
  static __device__ __forceinline__ void floats(const Raw& r, int K, float (&f)[EPT]) {  // 0 where they are not its own
    raw_to_floats<DT, NV * 4>(r.w, f);
    if constexpr (MODE == kLoose)
#pragma unroll
      for (int e = 0; e < EPT; ++e) f[e] = own(e, K) ? f[e] : 0.0f;
  }
  static __device__ __forceinline__ void store(const float (&f)[EPT], void* base, int64_t row, int K) {
    E* p = reinterpret_cast<E*>(base) + row * K;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (place(v) < K) store_vector<DT, VEC, MODE>(p + at(v, K), place(v) - at(v, K), K, f + v * VEC);
  }
  // a parameter of the thread's columns, `none` outside and where p is NULL
  static __device__ __forceinline__ void param(const void* p, const ResArgs& a, float none, float (&f)[NP]) {
    const E* q = reinterpret_cast<const E*>(p);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const bool mine = own(i * GR, a.K);
      const float v = p ? (float)q[mine ? channel_of(at(i * GR / VEC, a.K) + i * GR % VEC, a.mT) : 0] : none;
      f[i] = mine ? v : none;
    }
  }
  // the sum over a row's threads
  static __device__ __forceinline__ float total(float s, float* red, int& slot) {
    if constexpr (LANES < 16) {
      s += dpp<0xB1>(s);  // quad_perm 1 0 3 2, then 2 3 0 1
      s += dpp<0x4E>(s);
      if constexpr (LANES == 8) s += dpp<0x141>(s);  // half row mirrored: the other quad
    } else {
      s += dpp<0x128>(s);  // rows of 16 lanes rotated by 8, 4, 2, 1
      s += dpp<0x124>(s);
      s += dpp<0x122>(s);
      s += dpp<0x121>(s);
    }
    if constexpr (LANES >= 32) {
      float t = s;
      swap16(s, t);
      s += t;
    }
    if constexpr (LANES >= 64) {
      float t = s;
      swap32(s, t);
      s += t;
    }
    if constexpr (LANES > 64) {
      constexpr int NW = LANES / 64;
      float* const q = red + slot * NW;  // alternating, so that one barrier a sum is enough
      slot ^= 1;
      if ((threadIdx.x & 63) == 0) q[threadIdx.x >> 6] = s;
      __syncthreads();
      s = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; w += 2) s += q[w] + q[w + 1];
    }
    return s;
  }
  // s and the sum of f, or f h, over run i of columns; a run adds to s as one, which keeps the digits of many rows
  static __device__ __forceinline__ float values(const float (&f)[EPT], int i, float s) {
    float t = f[i * GR];
#pragma unroll
    for (int j = 1; j < GR; ++j) t += f[i * GR + j];
    return s + t;
  }
  static __device__ __forceinline__ float products(const float (&f)[EPT], const float (&h)[EPT], int i, float s) {
    if constexpr (GR == 1) return __builtin_fmaf(f[i], h[i], s);
    float t = f[i * GR] * h[i * GR];
#pragma unroll
    for (int j = 1; j < GR; ++j) t = __builtin_fmaf(f[i * GR + j], h[i * GR + j], t);
    return s + t;
  }
  // f normalised in place (0 outside the row); returns the factor
  static __device__ __forceinline__ float normed(float (&f)[EPT], const ResArgs& a, float* red, int& slot) {
    float s = 0.0f;
    if (!a.rms) {
#pragma unroll
      for (int e = 0; e < EPT; ++e) s += f[e];
      const float mean = total(s, red, slot) / (float)a.K;
#pragma unroll
      for (int e = 0; e < EPT; ++e) f[e] = own(e, a.K) ? f[e] - mean : 0.0f;
      s = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) s = __builtin_fmaf(f[e], f[e], s);
    const float k = 1.0f / sqrtf(total(s, red, slot) / (float)a.K + a.eps);
#pragma unroll
    for (int e = 0; e < EPT; ++e) f[e] *= k;
    return k;
  }
  // the gradient g of a normalised row through the norm, in place (0 outside the row)
  static __device__ __forceinline__ void back(float (&g)[EPT], const float (&f)[EPT], float k, const ResArgs& a, float* red,
                                              int& slot) {
    float s = 0.0f, m = 0.0f;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      s = __builtin_fmaf(g[e], f[e], s);
      m += g[e];
    }
    s = total(s, red, slot) / (float)a.K;
    m = a.rms ? 0.0f : total(m, red, slot) / (float)a.K;
#pragma unroll
    for (int e = 0; e < EPT; ++e)
      g[e] = own(e, a.K) ? k * (g[e] - __builtin_fmaf(f[e], s, m)) : 0.0f;
  }
};

// Strip of a workgroup: rows first + its own .. last of sequence q.
struct ResPlace {
  int64_t q, strip, first, last;
};
__device__ __forceinline__ ResPlace res_place(const ResArgs& a) {
  ResPlace p;
  const SlicePlace at = slice_place(a.seq, a.first, blockIdx.x, (unsigned)a.strips);
  p.q = at.seq;
  p.strip = at.at;
  p.first = p.strip * a.strip;
  p.last = min(p.first + a.strip, a.rows);
  return p;
}
// scale[c] gate[q, c] of the thread's columns
template <typename R>
__device__ __forceinline__ void res_scale(const ResArgs& a, const ResPlace& p, float (&k)[R::NP]) {
  R::param(a.scale, a, 1.0f, k);
  if (!a.gate) return;
  float g[R::NP];
  R::param(reinterpret_cast<const typename R::E*>(a.gate) + p.q * a.C, a, 1.0f, g);
#pragma unroll
  for (int i = 0; i < R::NP; ++i) k[i] *= g[i];
}

template <int DT, int LANES, int EPT, int MODE, int GR>
__global__ __launch_bounds__((ResRow<DT, LANES, EPT, MODE, GR>::THREADS)) void eql_res_fwd_kernel(const ResArgs a) {
  using R = ResRow<DT, LANES, EPT, MODE, GR>;
  __shared__ float red[2 * (LANES > 64 ? LANES / 64 : 1)];
  const ResPlace p = res_place(a);
  int slot = 0;
  const int mine = LANES < 256 ? threadIdx.x / LANES : 0;
  typename R::Raw xr, ur;
  auto fetch = [&](int64_t row) {
    R::load(xr, a.x, p.q * a.rows + row, a.K, row < p.last);
    if (a.u) R::load(ur, a.u, p.q * a.rows + row, a.K, row < p.last);
  };
  fetch(p.first + mine);
  float k[R::NP], w[R::NP], b[R::NP], pw[R::NP], pb[R::NP];
  res_scale<R>(a, p, k);
  R::param(a.w, a, 0.0f, w);
  R::param(a.b, a, 0.0f, b);
  R::param(a.pw, a, 0.0f, pw);
  R::param(a.pb, a, 0.0f, pb);
  // (LANES > 64: one row a workgroup, so every thread takes every turn)
  for (int64_t i = p.first + mine; i < p.last; i += R::ROWS) {
    const int64_t row = p.q * a.rows + i;
    float x[EPT], u[EPT];
    R::floats(xr, a.K, x);
    if (a.u) R::floats(ur, a.K, u);
    if (i + R::ROWS < p.last) fetch(i + R::ROWS);
    if (a.u) {
      if (a.pw) {
        R::normed(u, a, red, slot);
#pragma unroll
        for (int e = 0; e < EPT; ++e) u[e] = __builtin_fmaf(u[e], pw[e / GR], pb[e / GR]);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) x[e] = __builtin_fmaf(k[e / GR], u[e], x[e]);
      R::store(x, a.r, row, a.K);
    }
    if (a.w) {
      R::normed(x, a, red, slot);
#pragma unroll
      for (int e = 0; e < EPT; ++e) x[e] = __builtin_fmaf(x[e], w[e / GR], b[e / GR]);
      R::store(x, a.h, row, a.K);
    }
  }
}

// Rows of column sums: dw, db (where there is a norm after), then E, or P and S.
template <int DT, int LANES, int EPT, int MODE, int GR>
__global__ __launch_bounds__((ResRow<DT, LANES, EPT, MODE, GR>::THREADS)) void eql_res_bwd_kernel(const ResArgs a) {
  using R = ResRow<DT, LANES, EPT, MODE, GR>;
  constexpr int NP = R::NP;
  __shared__ float red[2 * (LANES > 64 ? LANES / 64 : 1)];
  __shared__ float cols[R::ROWS > 1 ? R::ROWS * LANES * NP : 1];
  // Parameters of a thread's own in LDS where 1024 threads leave each 128 registers: a row's are read as it needs them
  // (kept in registers they go to scratch memory with every row).
  constexpr bool PARK = LANES == 1024 && GR == 1;
  __shared__ floatx4 parked[PARK ? NP * LANES : 1];
  auto park = [&](int j, const float (&f)[NP]) {
    if constexpr (PARK)
#pragma unroll
      for (int i = 0; i < NP; i += 4) parked[(j * NP + i) / 4 * LANES + threadIdx.x] = floatx4{f[i], f[i + 1], f[i + 2], f[i + 3]};
  };
  auto again = [&](int j, float (&f)[NP]) {
    if constexpr (PARK)
#pragma unroll
      for (int i = 0; i < NP; i += 4) {
        const floatx4 v = parked[(j * NP + i) / 4 * LANES + threadIdx.x];
#pragma unroll
        for (int o = 0; o < 4; ++o) f[i + o] = v[o];
      }
  };
  const ResPlace p = res_place(a);
  int slot = 0;
  const int mine = LANES < 256 ? threadIdx.x / LANES : 0;
  typename R::Raw xr, ur, rr, hr;
  auto fetch = [&](int64_t i) {
    const int64_t row = p.q * a.rows + i;
    const bool on = i < p.last;
    R::load(xr, a.x, row, a.K, on);
    if (a.u) R::load(ur, a.u, row, a.K, on);
    if (a.dh) R::load(hr, a.dh, row, a.K, on);
    if (a.dr) R::load(rr, a.dr, row, a.K, on);
  };
  if (!PARK) fetch(p.first + mine);  // (PARK: no registers for two rows)
  float k[NP], w[NP], pw[NP], pb[NP];
  res_scale<R>(a, p, k);
  R::param(a.w, a, 0.0f, w);
  R::param(a.pw, a, 0.0f, pw);
  R::param(a.pb, a, 0.0f, pb);
  park(0, k);
  park(1, w);
  park(2, pw);
  park(3, pb);
  float s0[NP], s1[NP], s2[NP], s3[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) s0[i] = s1[i] = s2[i] = s3[i] = 0.0f;
  for (int64_t i = p.first + mine; i < p.last; i += R::ROWS) {
    const int64_t row = p.q * a.rows + i;
    float x[EPT], u[EPT], g[EPT], d[EPT], fu = 1.0f;
    if (PARK) fetch(i);
    R::floats(xr, a.K, x);
    if (a.u) R::floats(ur, a.K, u);
    if (a.dh && !PARK) R::floats(hr, a.K, g);
    if (a.dr && !PARK) R::floats(rr, a.K, d);
    if (!PARK && i + R::ROWS < p.last) fetch(i + R::ROWS);
    if (a.u) {
      again(0, k);
      if (a.pw) {
        again(2, pw);
        again(3, pb);
        fu = R::normed(u, a, red, slot);  // u: uh
#pragma unroll
        for (int e = 0; e < EPT; ++e) x[e] = __builtin_fmaf(k[e / GR], __builtin_fmaf(u[e], pw[e / GR], pb[e / GR]), x[e]);
      } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) x[e] = __builtin_fmaf(k[e / GR], u[e], x[e]);
      }
    }
    if (a.dh) {
      const float fr = R::normed(x, a, red, slot);  // x: rh
      again(1, w);
      if (PARK) R::floats(hr, a.K, g);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        s0[i] = R::products(g, x, i, s0[i]);
        s1[i] = R::values(g, i, s1[i]);
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) g[e] *= w[e / GR];
      R::back(g, x, fr, a, red, slot);
      if (a.dr && PARK) R::floats(rr, a.K, d);
      if (a.dr)
#pragma unroll
        for (int e = 0; e < EPT; ++e) g[e] += d[e];
    } else {
      if (a.dr && PARK) R::floats(rr, a.K, d);
#pragma unroll
      for (int e = 0; e < EPT; ++e) g[e] = a.dr ? d[e] : 0.0f;
    }
    if (a.dx) R::store(g, a.dx, row, a.K);
    if (a.u) {
#pragma unroll
      for (int i = 0; i < NP; ++i) s2[i] = R::products(g, u, i, s2[i]);
      again(0, k);
      if (a.pw) {
        again(2, pw);
#pragma unroll
        for (int i = 0; i < NP; ++i) s3[i] = R::values(g, i, s3[i]);
#pragma unroll
        for (int e = 0; e < EPT; ++e) g[e] *= k[e / GR] * pw[e / GR];
        if (a.du) R::back(g, u, fu, a, red, slot);
      } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) g[e] *= k[e / GR];
      }
      if (a.du) R::store(g, a.du, row, a.K);
    }
  }
  const int K = a.K / GR;  // columns of the sums
  float* const part = a.part + (p.q * a.strips + p.strip) * a.J * K;
  int j = 0;
  auto put = [&](const float (&s)[NP]) {
    if constexpr (R::ROWS > 1) {
      if (j) __syncthreads();
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (R::at(i * GR / R::VEC, a.K) + i * GR % R::VEC) / GR;
        if (R::own(i * GR, a.K)) cols[mine * (LANES * NP) + c] = s[i];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < K; c += R::THREADS) {
        float v = cols[c];
#pragma unroll
        for (int m = 1; m < R::ROWS; ++m) v += cols[m * (LANES * NP) + c];
        part[(int64_t)j * K + c] = v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int c = (R::at(i * GR / R::VEC, a.K) + i * GR % R::VEC) / GR;
        if (R::own(i * GR, a.K)) part[(int64_t)j * K + c] = s[i];
      }
    }
    ++j;
  };
  if (a.w) {
    put(s0);
    put(s1);
  }
  if (a.u) {
    put(s2);
    if (a.pw) put(s3);
  }
}

// sums[q, j, c]: the strips and group elements of a sequence's column sums.
template <int UNUSED = 0>
__global__ __launch_bounds__(kColsumThreads) void eql_res_strips_kernel(const ResArgs a, int GR, int blocks) {
  const SlicePlace at = slice_place(a.seq, a.first, blockIdx.x, (unsigned)(a.J * blocks));
  const int block = (int)(at.at % (unsigned)blocks), j = (int)(at.at / (unsigned)blocks), T = a.T / GR, K = a.K / GR;
  const int64_t q = at.seq;
  column_sums(a.part + (q * a.strips * a.J + j) * K, a.strips, (int64_t)a.J * K, a.C, T, block,
              [&](int c, float v) { a.sums[(q * a.J + j) * a.C + c] = v; });
}
// The parameters' gradients: a workgroup takes 16 channels, its 64 threads of each every 64th sequence.
constexpr int kResParamThreads = 1024, kResParamChannels = 16;
template <int DT>
__global__ __launch_bounds__(kResParamThreads) void eql_res_params_kernel(const ResArgs a) {
  using E = typename Elem<DT>::T;
  constexpr int NC = kResParamChannels, NQ = kResParamThreads / NC;
  const int cc = threadIdx.x % NC, turn = threadIdx.x / NC, c = (int)blockIdx.x * NC + cc;
  __shared__ float red[5][NQ][NC];
  auto at = [&](const void* p, int64_t i) { return (float)reinterpret_cast<const E*>(p)[i]; };
  float sum[5] = {0.f, 0.f, 0.f, 0.f, 0.f};  // dw, db, dscale, dpw, dpb
  float many[5] = {0.f, 0.f, 0.f, 0.f, 0.f};  // of 64 sequences each, so that thousands lose no digits
  int turns = 0;
  if (c < a.C) {
    const float scale = a.scale ? at(a.scale, c) : 1.0f, pw = a.pw ? at(a.pw, c) : 1.0f, pb = a.pb ? at(a.pb, c) : 0.0f;
    for (int64_t q = turn; q < a.seqs; q += NQ) {
      if (a.rows == 0) {  // no tokens: nothing was summed
        if (a.dgate) reinterpret_cast<E*>(a.dgate)[q * a.C + c] = (E)0.0f;
        continue;
      }
      const float* s = a.sums + q * a.J * a.C + c;
      if (++turns == 64) {
        turns = 0;
#pragma unroll
        for (int i = 0; i < 5; ++i) {
          many[i] += sum[i];
          sum[i] = 0.0f;
        }
      }
      if (a.w) {
        sum[0] += s[0];
        sum[1] += s[a.C];
        s += 2 * a.C;
      }
      if (!a.u) continue;
      const float gate = a.gate ? at(a.gate, q * a.C + c) : 1.0f, P = s[0], S = a.pw ? s[a.C] : 0.0f;
      const float e = a.pw ? __builtin_fmaf(pw, P, pb * S) : P;
      if (a.dgate) reinterpret_cast<E*>(a.dgate)[q * a.C + c] = (E)(scale * e);
      sum[2] = __builtin_fmaf(gate, e, sum[2]);
      sum[3] = __builtin_fmaf(gate * scale, P, sum[3]);
      sum[4] = __builtin_fmaf(gate * scale, S, sum[4]);
    }
  }
#pragma unroll
  for (int i = 0; i < 5; ++i) red[i][turn][cc] = many[i] + sum[i];
  __syncthreads();
  if (c >= a.C || turn >= 5) return;
  void* const dst[5] = {a.dw, a.db, a.dscale, a.dpw, a.dpb};
  float v = 0.0f;
#pragma unroll 8
  for (int q = 0; q < NQ; ++q) v += red[turn][q][cc];
  void* p = nullptr;
#pragma unroll
  for (int i = 0; i < 5; ++i) p = turn == i ? dst[i] : p;
  if (p) reinterpret_cast<E*>(p)[c] = (E)v;
}

}  // namespace eqk
