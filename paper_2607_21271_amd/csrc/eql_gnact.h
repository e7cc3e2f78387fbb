// eql_gnact.h -- group norm with an activation over channels-last features
// x [B, S, C, T] (K = C T contiguous elements a position), for gfx950:
//   z = (x - mean) rstd w[c] + b[c],  y = act(z),
// mean and variance of a sequence's S positions, C / G channels and T group
// elements, so that the map commutes with the group action.
//
// Groups that fit the registers of a workgroup (up to 128 K 16-bit values forward, 64 K
// backward) take one kernel that reads everything once; the others two passes.
// Every pass gives a thread VEC fixed columns of the K and lets it walk the
// positions of its workgroup's chunk, so weights and statistics are registers
// and column sums need no exchange until the end.  Forward: mean and squared deviations
// per chunk and group, then the map, whose workgroups join the chunks' in order.  Every
// sum of squares is taken about a value of its own few elements (a column's first, then a
// mean) and moved to the mean of what it joins: one value far from all others, the first
// of a padded image say, costs no more than its own column's last bits.  Backward: channel sums of dz and dz xhat per chunk, one
// small kernel that adds the chunks, then dx together with dw and db.
//
// Bound: memory, and with gelu in 16 bits the vector pipe as much (about 30 operations
// an element, twice in the backward).  Held groups, 128 x 3136 x 96 fp16, silu: 42 us, 3.7 TB/s (two
// workgroups of 1,024 threads a CU load, compute and store at the same time as one
// another; in two passes over memory 45 us); 32 x 784 x 256 bf16, gelu: forward 15 us, backward 27 + 4
// (in passes 22 and 33).  In passes, silu in fp16: 8 x 50,176 x 24 x 4 46 us, 3.4 TB/s with the host.
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
  float* part;    // forward [B, P, G, 2] mean, squared deviations; backward [B, chunks, C, 2]
  float* sums;    // backward [B, C, 2]: sums of dz xhat and dz
  int64_t B, S;
  int C, T, G, K, act;
  float eps;
  int chunks, cblocks, rows;  // chunks of `rows` positions, blocks of `width` vectors of columns
  int width;                  // at most 256, whole channels
  int hold;                   // vectors a thread holds where a workgroup holds a group, else 0
  int threads;                // of such a workgroup
};

// The normal distribution's cdf and exp(-z^2 / 2) at z.  16-bit types: erf by
// Abramowitz and Stegun 7.1.26, |error| <= 1.5e-7; its exponential is the density's.
// z cdf is then at most 2.1e-7 off beside fp32's own rounding: below a quarter of a unit of a 16-bit
// result from 2e-3 on, in the tail of negative z up to one unit of fp16; of bf16 one to z = -6, three to
// -8 and ten to -13, results of less than 1e-8 and 1e-14.  Full precision takes the library function.
template <int DT>
__device__ __forceinline__ void gn_normal(float z, float& cdf, float& e) {
  if constexpr (DT == kF32) {
    e = expf(-0.5f * z * z);
    cdf = 0.5f * (1.0f + erff(z * 0.70710678118654752f));
  } else {
    const float x = __builtin_fabsf(z) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
    float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
    p = __builtin_fmaf(p, t, 1.421413741f);
    p = __builtin_fmaf(p, t, -0.284496736f);
    p = __builtin_fmaf(p, t, 0.254829592f);
    const float tail = 0.5f * p * t * e;  // of |z|
    cdf = z < 0.0f ? tail : 1.0f - tail;
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
  else if constexpr (ACT == kActGelu) {
    float cdf, e;
    gn_normal<DT>(z, cdf, e);
    return z * cdf;
  } else return z;
}
template <int DT, int ACT>
__device__ __forceinline__ float gn_dact(float z) {
  if constexpr (ACT == kActRelu) {
    return z > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == kActSilu) {
    const float s = gn_sigmoid<DT>(z);
    return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
  } else if constexpr (ACT == kActGelu) {
    float cdf, e;
    gn_normal<DT>(z, cdf, e);
    return __builtin_fmaf(z * 0.39894228040143268f, e, cdf);
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
// rows first, first + step, ... below last; ch, t and grp are those of col0.
struct GnPlace {
  int64_t b, first, last;
  int chunk, cb, step, rr, cv, col0, cols;  // cols: columns of the block
  int ch, t, grp;
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
  const int nvb = min(nv - p.cb * a.width, a.width);
  p.step = 256 / nvb;
  p.rr = threadIdx.x / nvb;
  p.cv = threadIdx.x % nvb;
  p.on = p.rr < p.step;
  p.col0 = (p.cb * a.width + p.cv) * VEC;
  p.cols = nvb * VEC;
  p.ch = (unsigned)p.col0 / (unsigned)a.T;
  p.t = p.col0 - p.ch * a.T;
  p.grp = (unsigned)p.ch / (unsigned)(a.C / a.G);
  p.first = (int64_t)p.chunk * a.rows + p.rr;
  p.last = min((int64_t)(p.chunk + 1) * a.rows, a.S);
  return p;
}
// f(k, channel, group) for the thread's columns col0 + k
template <int VEC, typename F>
__device__ __forceinline__ void gn_columns(const GnArgs& a, const GnPlace& p, F&& f) {
  const int cg = a.C / a.G;
  int ch = p.ch, t = p.t, g = p.grp, next = (g + 1) * cg;
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    f(k, ch, g);
    if (++t == a.T) {
      t = 0;
      if (++ch == next) {
        ++g;
        next += cg;
      }
    }
  }
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
  // a column of the thread: its sums of x - x0 and the square, x0 its first element
  const int have = (int)(p.last - (int64_t)p.chunk * a.rows);  // rows of the chunk
  const int each = have / p.step, more = have - each * p.step;
  auto rows_of = [&](int rr) { return each + (rr < more ? 1 : 0); };
  float s1[VEC], s2[VEC], x0[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) s1[k] = s2[k] = x0[k] = 0.0f;
  if (p.on && p.first < p.last) {
    const V v0 = *(const V*)(xb + p.first * a.K + p.col0);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x0[k] = (float)v0.e[k];
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
    const float inv = p.first < p.last ? 1.0f / (float)rows_of(p.rr) : 0.0f;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float d = s1[k] * inv;
      red[0][p.rr * p.cols + p.cv * VEC + k] = x0[k] + d;
      red[1][p.rr * p.cols + p.cv * VEC + k] = __builtin_fmaf(-d, s1[k], s2[k]);
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 63, c0 = p.cb * a.width * VEC;
  float* const out = a.part + ((p.b * a.chunks + p.chunk) * a.cblocks + p.cb) * a.G * 2;
  for (int g = threadIdx.x >> 6; g < a.G; g += 4) {
    const int lo = max(g * gw, c0) - c0, hi = min((g + 1) * gw, c0 + p.cols) - c0;
    float t1 = 0.0f, t2 = 0.0f;
    const int w = hi - lo;
    const float ref = w > 0 ? red[0][lo] : 0.0f;
    for (int i = lane; i < w * p.step; i += 64) {
      const int rr = i / w, at = rr * p.cols + lo + i % w;
      const float d = red[0][at] - ref, n = (float)rows_of(rr);
      if (n > 0.0f) {
        t1 = __builtin_fmaf(n, d, t1);
        t2 += __builtin_fmaf(n * d, d, red[1][at]);
      }
    }
    t1 = wave_sum(t1);
    t2 = wave_sum(t2);
    if (lane == 0) {
      const float d = w > 0 ? t1 / ((float)have * (float)w) : 0.0f;
      out[2 * g] = ref + d;
      out[2 * g + 1] = __builtin_fmaf(-d, t1, t2);
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
    // the parts' sums about the group's first part: `lanes` threads a group each add every
    // lanes-th part, then the threads of a group in order
    const float inv = 1.0f / ((float)a.S * (float)gw);
    const float2* const part = (const float2*)a.part + p.b * parts * a.G;
    __shared__ float2 add[256];
    const int gs = min(a.G, 256), lanes = 256 / gs, bw = a.width * VEC;
    for (int g0 = 0; g0 < a.G; g0 += gs) {
      const int g = g0 + (int)threadIdx.x % gs, l = threadIdx.x / gs;
      float t1 = 0.0f, t2 = 0.0f, ref = 0.0f;
      if (g < a.G && l < lanes) {
        ref = part[g * gw / bw * a.G + g].x;
        // part i is block cb of its chunk; the parts of the last chunk, from `short_from` on, hold fewer rows
        int cb = l % a.cblocks;
        const int turn = lanes % a.cblocks, short_from = parts - a.cblocks;
        const float full = (float)a.rows, rest = (float)(int)(a.S - (int64_t)(a.chunks - 1) * a.rows);
#pragma unroll 4
        for (int i = l; i < parts; i += lanes) {
          const float2 v = part[i * a.G + g];
          const int c0 = cb * bw, w = min((g + 1) * gw, c0 + bw) - max(g * gw, c0);  // columns of the group in the part
          const float n = w > 0 ? (float)w * (i < short_from ? full : rest) : 0.0f;
          cb += turn;
          cb -= cb >= a.cblocks ? a.cblocks : 0;
          const float d = w > 0 ? v.x - ref : 0.0f;
          t1 = __builtin_fmaf(n, d, t1);
          t2 += __builtin_fmaf(n * d, d, v.y);
        }
        add[threadIdx.x] = make_float2(t1, t2);
      }
      __syncthreads();
      // sixteen neighbours of a group's threads at a time where there are many
      for (int w = 16; w < lanes; w *= 16) {
        if (g < a.G && l < lanes && l % w == 0) {
          const int s = w / 16;
          t1 = t2 = 0.0f;
          for (int i = 0; i < 16 && l + i * s < lanes; ++i) {
            const float2 v = add[(l + i * s) * gs + (int)threadIdx.x % gs];
            t1 += v.x;
            t2 += v.y;
          }
        }
        __syncthreads();
        if (g < a.G && l < lanes && l % w == 0) add[threadIdx.x] = make_float2(t1, t2);
        __syncthreads();
      }
      if (g < a.G && l == 0) {
        int w = 1;
        while (w * 16 < lanes) w *= 16;
        t1 = t2 = 0.0f;
        for (int i = 0; i < lanes; i += w) {
          const float2 v = add[i * gs + threadIdx.x];
          t1 += v.x;
          t2 += v.y;
        }
        t1 *= inv;
        t2 *= inv;
        const float var = __builtin_fmaf(-t1, t1, t2);
        const float mean = ref + t1, rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + a.eps);
        st[g] = make_float2(mean, rstd);
        if (a.stats && p.chunk == 0 && p.cb == 0) {
          a.stats[(p.b * a.G + g) * 2] = mean;
          a.stats[(p.b * a.G + g) * 2 + 1] = rstd;
        }
      }
      __syncthreads();
    }
  }
  __syncthreads();
  if (!p.on) return;
  float mu[VEC], m[VEC], c[VEC];
  gn_columns<VEC>(a, p, [&](int k, int ch, int g) {
    const float2 s = st[g];
    mu[k] = s.x;
    m[k] = s.y * (float)((const E*)a.w)[ch];
    c[k] = (float)((const E*)a.b)[ch];
  });
  E* const yb = (E*)a.y + p.b * a.S * a.K;
#pragma unroll 4
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
  const E* const xb = (const E*)a.x + p.b * a.S * a.K;
  const E* const gb = (const E*)a.dy + p.b * a.S * a.K;
  float s1[VEC], s2[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) s1[k] = s2[k] = 0.0f;
  if (p.on) {
    float mu[VEC], rs[VEC], w[VEC], c[VEC];
    gn_columns<VEC>(a, p, [&](int k, int ch, int g) {
      const float2 s = ((const float2*)a.stats)[p.b * a.G + g];
      mu[k] = s.x;
      rs[k] = s.y;
      w[k] = (float)((const E*)a.w)[ch];
      c[k] = (float)((const E*)a.b)[ch];
    });
#pragma unroll 4
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
  // a block holds whole channels: every thread adds one channel's rows and group elements
  const int nch = p.cols / a.T, ch0 = p.cb * a.width * VEC / a.T;
  float2* const out = (float2*)a.part + (p.b * a.chunks + p.chunk) * a.C + ch0;
  for (int i = threadIdx.x; i < nch; i += 256) {
    float t1 = 0.0f, t2 = 0.0f;
    for (int r = 0; r < p.step; ++r)
      for (int t = 0; t < a.T; ++t) {
        t1 += red[0][r * p.cols + i * a.T + t];
        t2 += red[1][r * p.cols + i * a.T + t];
      }
    out[i] = make_float2(t1, t2);
  }
}

// Adds the chunks of one sequence's channels: 64 channels a workgroup, each by four
// threads that take every fourth chunk.
static __global__ __launch_bounds__(256) void eql_gn_bchunks_kernel(GnArgs a) {
  __shared__ float2 add[256];
  const uint32_t tiles = (uint32_t)(a.C + 63) / 64;
  const int64_t b = blockIdx.x / tiles;
  const int c = (int)(blockIdx.x % tiles) * 64 + (threadIdx.x & 63);
  const float2* const part = (const float2*)a.part + b * a.chunks * a.C + c;
  float t1 = 0.0f, t2 = 0.0f;
  if (c < a.C) {
#pragma unroll 8
    for (int q = threadIdx.x >> 6; q < a.chunks; q += 4) {
      const float2 v = part[(int64_t)q * a.C];
      t1 += v.x;
      t2 += v.y;
    }
  }
  add[threadIdx.x] = make_float2(t1, t2);
  __syncthreads();
  if (threadIdx.x >= 64 || c >= a.C) return;
  for (int i = 64; i < 256; i += 64) {
    t1 += add[i + threadIdx.x].x;
    t2 += add[i + threadIdx.x].y;
  }
  ((float2*)a.sums)[b * a.C + c] = make_float2(t1, t2);
}

// dw and db: the sequences' sums of a channel, one wave each.
template <int DT>
__device__ __forceinline__ void gn_params(const GnArgs& a, int c) {
  using E = typename Elem<DT>::T;
  const int lane = threadIdx.x & 63;
  if (c >= a.C) return;
  float t1 = 0.0f, t2 = 0.0f;
  for (int64_t b = lane; b < a.B; b += 64) {
    const float2 v = ((const float2*)a.sums)[b * a.C + c];
    t1 += v.x;
    t2 += v.y;
  }
  t1 = wave_sum(t1);
  t2 = wave_sum(t2);
  if (lane == 0) {
    ((E*)a.dw)[c] = (E)t1;
    ((E*)a.db)[c] = (E)t2;
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
    gn_params<DT>(a, (int)(blockIdx.x - main) * 4 + (threadIdx.x >> 6));
    return;
  }
  const GnPlace p = gn_place<VEC>(a, blockIdx.x);
  __shared__ float2 means[kGnMaxGroups];  // of w dz xhat and w dz
  {
    const int lane = threadIdx.x & 63, cg = a.C / a.G;
    const float inv = 1.0f / ((float)a.S * (float)(a.K / a.G));
    const float2* const sums = (const float2*)a.sums + p.b * a.C;
    // `lanes` neighbours of a wave a group: a power of two, at least the channels where they fit
    int lanes = 1;
    while (lanes < cg && lanes < 64) lanes *= 2;
    for (int g0 = 0; g0 < a.G; g0 += 256 / lanes) {
      const int g = g0 + (int)threadIdx.x / lanes;
      float t1 = 0.0f, t2 = 0.0f;
      if (g < a.G)
        for (int i = lane % lanes; i < cg; i += lanes) {
          const float2 v = sums[g * cg + i];
          const float w = (float)((const E*)a.w)[g * cg + i];
          t1 = __builtin_fmaf(w, v.x, t1);
          t2 = __builtin_fmaf(w, v.y, t2);
        }
      for (int d = 1; d < lanes; d *= 2) {
        t1 += __shfl_xor(t1, d);
        t2 += __shfl_xor(t2, d);
      }
      if (g < a.G && lane % lanes == 0) means[g] = make_float2(t1 * inv, t2 * inv);
    }
  }
  __syncthreads();
  if (!p.on) return;
  const int64_t base = p.b * a.S * a.K;
  const E *const xb = (const E*)a.x + base, *const gb = (const E*)a.dy + base;
  E* const ob = (E*)a.dx + base;
  float mu[VEC], rs[VEC], w[VEC], c[VEC], m1[VEC], m2[VEC];
  gn_columns<VEC>(a, p, [&](int k, int ch, int g) {
    const float2 s = ((const float2*)a.stats)[p.b * a.G + g], m = means[g];
    mu[k] = s.x;
    rs[k] = s.y;
    m1[k] = m.x;
    m2[k] = m.y;
    w[k] = (float)((const E*)a.w)[ch];
    c[k] = (float)((const E*)a.b)[ch];
  });
#pragma unroll 4
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

// ---- groups that one workgroup holds -----------------------------------------
// A workgroup keeps its group of one sequence in registers: NT threads, each at most R
// 16-byte vectors of fixed columns, so x (and dy) are read once and statistics are two
// passes over registers.  Consecutive workgroups of an XCD take the groups of one
// sequence, whose rows share cache lines.
struct GnHold {
  int64_t b;
  int g, vpg, rpp, c, r0;
  int64_t at;  // element of the thread's first vector
  bool on;
};
template <int VEC, int NT>
__device__ __forceinline__ GnHold gn_hold(const GnArgs& a) {
  GnHold h;
  const uint32_t n = gridDim.x, q = n / 8, rest = n % 8, xcd = blockIdx.x % 8;
  const uint32_t id = xcd * q + min(xcd, rest) + blockIdx.x / 8;
  h.b = id / (uint32_t)a.G;
  h.g = (int)(id % (uint32_t)a.G);
  h.vpg = a.K / a.G / VEC;
  h.rpp = NT / h.vpg;
  h.c = (int)threadIdx.x % h.vpg;
  h.r0 = (int)threadIdx.x / h.vpg;
  h.on = h.r0 < h.rpp;
  h.at = (h.b * a.S + h.r0) * a.K + (int64_t)h.g * (a.K / a.G) + h.c * VEC;
  return h;
}
// Sum over the workgroup, the same in every thread; `red` of NT / 64 floats of its own.
template <int NT>
__device__ __forceinline__ float gn_total(float v, float* red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) t += red[w];
  return t;
}
// f(k, channel of column k of the thread) where T elements make a channel
template <int VEC, typename F>
__device__ __forceinline__ void gn_hold_columns(const GnArgs& a, const GnHold& h, F&& f) {
  int ch = h.c * VEC / a.T, t = h.c * VEC - ch * a.T;
  ch += h.g * (a.C / a.G);
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    f(k, ch);
    if (++t == a.T) {
      t = 0;
      ++ch;
    }
  }
}

// The elements of a held vector.  The compiler may not keep their conversions from one
// pass over the registers to the next: twice the registers, spilled.
template <typename V>
__device__ __forceinline__ V gn_words(u32x4& w) {
  asm volatile("" : "+v"(w));
  return __builtin_bit_cast(V, w);
}

template <int DT, int ACT, int NT, int R>
__global__ __launch_bounds__(NT) void eql_gn_hold_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  constexpr int VEC = DT == kF32 ? 4 : 8;
  using V = typename GnVec<DT, VEC>::V;
  __shared__ float red[2][NT / 64];
  const GnHold h = gn_hold<VEC, NT>(a);
  const int64_t step = (int64_t)h.rpp * a.K;
  const int rows = h.on ? (int)((a.S - h.r0 + h.rpp - 1) / h.rpp) : 0;  // of the thread
  const E* const x = (const E*)a.x + h.at;
  // sums of x - x0, x0 the group's first element: exact however far the mean lies from zero
  const float x0 = (float)((const E*)a.x)[h.b * a.S * a.K + (int64_t)h.g * (a.K / a.G)];
  u32x4 v[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) v[i] = *(const u32x4*)(x + i * step);
  const float inv = 1.0f / ((float)a.S * (float)(a.K / a.G));
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) {
      const V e = gn_words<V>(v[i]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) s += (float)e.e[k] - x0;
    }
  const float mean = x0 + gn_total<NT>(s, red[0]) * inv;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) {
      const V e = gn_words<V>(v[i]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float d = (float)e.e[k] - mean;
        s = __builtin_fmaf(d, d, s);
      }
    }
  const float rstd = 1.0f / sqrtf(gn_total<NT>(s, red[1]) * inv + a.eps);
  if (a.stats && threadIdx.x == 0) ((float2*)a.stats)[h.b * a.G + h.g] = make_float2(mean, rstd);
  float m[VEC], c[VEC];
  gn_hold_columns<VEC>(a, h, [&](int k, int ch) {
    m[k] = h.on ? rstd * (float)((const E*)a.w)[ch] : 0.0f;
    c[k] = h.on ? (float)((const E*)a.b)[ch] : 0.0f;
  });
  E* const y = (E*)a.y + h.at;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) {
      V e = gn_words<V>(v[i]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) e.e[k] = (E)gn_act<DT, ACT>(__builtin_fmaf((float)e.e[k] - mean, m[k], c[k]));
      *(V*)(y + i * step) = e;
    }
}

template <int DT, int ACT, int NT, int R>
__global__ __launch_bounds__(NT) void eql_gn_bhold_kernel(GnArgs a) {
  using E = typename Elem<DT>::T;
  constexpr int VEC = DT == kF32 ? 4 : 8;
  using V = typename GnVec<DT, VEC>::V;
  __shared__ float col[2][NT * VEC];
  __shared__ float red[2][NT / 64];
  const GnHold h = gn_hold<VEC, NT>(a);
  const int64_t step = (int64_t)h.rpp * a.K;
  const int rows = h.on ? (int)((a.S - h.r0 + h.rpp - 1) / h.rpp) : 0;
  const E *const x = (const E*)a.x + h.at, *const gy = (const E*)a.dy + h.at;
  u32x4 v[R], g[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) {
      v[i] = *(const u32x4*)(x + i * step);
      g[i] = *(const u32x4*)(gy + i * step);
    }
  const float2 st = ((const float2*)a.stats)[h.b * a.G + h.g];
  const float mu = st.x, rs = st.y;
  float w[VEC], c[VEC], s1[VEC], s2[VEC];
  gn_hold_columns<VEC>(a, h, [&](int k, int ch) {
    w[k] = h.on ? (float)((const E*)a.w)[ch] : 0.0f;
    c[k] = h.on ? (float)((const E*)a.b)[ch] : 0.0f;
    s1[k] = s2[k] = 0.0f;
  });
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) {
      const V e = gn_words<V>(v[i]), d = gn_words<V>(g[i]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float xh = ((float)e.e[k] - mu) * rs;
        const float dz = (float)d.e[k] * gn_dact<DT, ACT>(__builtin_fmaf(xh, w[k], c[k]));
        s1[k] = __builtin_fmaf(dz, xh, s1[k]);
        s2[k] += dz;
      }
    }
  // columns over the rows of threads, halves onto halves
  const int width = h.vpg * VEC, me = h.r0 * width + h.c * VEC;
  int half = 1;
  while (half < h.rpp) half *= 2;
  if (h.on) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      col[0][me + k] = s1[k];
      col[1][me + k] = s2[k];
    }
  }
  for (half /= 2; half > 0; half /= 2) {
    __syncthreads();
    if (h.r0 < half && h.r0 + half < h.rpp) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        col[0][me + k] += col[0][me + half * width + k];
        col[1][me + k] += col[1][me + half * width + k];
      }
    }
  }
  __syncthreads();
  // channels over T, and the group's means
  const int cg = a.C / a.G;
  float m1 = 0.0f, m2 = 0.0f;
  for (int i = threadIdx.x; i < cg; i += NT) {
    float t1 = 0.0f, t2 = 0.0f;
    for (int t = 0; t < a.T; ++t) {
      t1 += col[0][i * a.T + t];
      t2 += col[1][i * a.T + t];
    }
    const int ch = h.g * cg + i;
    ((float2*)a.sums)[h.b * a.C + ch] = make_float2(t1, t2);
    const float wc = (float)((const E*)a.w)[ch];
    m1 = __builtin_fmaf(wc, t1, m1);
    m2 = __builtin_fmaf(wc, t2, m2);
  }
  const float inv = 1.0f / ((float)a.S * (float)(a.K / a.G));
  m1 = gn_total<NT>(m1, red[0]) * inv;
  m2 = gn_total<NT>(m2, red[1]) * inv;
  E* const dx = (E*)a.dx + h.at;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (i < rows) {
      V e = gn_words<V>(v[i]);
      const V d = gn_words<V>(g[i]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float xh = ((float)e.e[k] - mu) * rs;
        const float dz = (float)d.e[k] * gn_dact<DT, ACT>(__builtin_fmaf(xh, w[k], c[k]));
        e.e[k] = (E)(rs * (__builtin_fmaf(-xh, m1, __builtin_fmaf(w[k], dz, -m2))));
      }
      *(V*)(dx + i * step) = e;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void eql_gn_params_kernel(GnArgs a) {
  gn_params<DT>(a, (int)blockIdx.x * 4 + (threadIdx.x >> 6));
}

}  // namespace eqk
