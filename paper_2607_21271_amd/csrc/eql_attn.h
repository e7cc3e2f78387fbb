// eql_attn.h -- attention with a sliding window and first tokens that stay
// visible, for gfx950: forward, forward over few rows split along the keys, and
// the two backward passes.
//
// Rows.  The G query heads that share a key/value head are taken together:
// packed row r of (sequence b, key/value head hk) is query token r / G of head
// hk G + r % G, R = Lq G rows in all.  Token i stands at position p = start + i
// and sees key j iff p < len, j < len, j <= p + right and (j >= p - left or
// j < sinks); a row that sees nothing gives zeros.
//
// Products.  All kernels compute transposed tiles with one owner a lane: in a
// 32 x 32 MFMA result a lane holds 16 entries of column lane % 32, entry e in
// row 8 (e / 4) + 4 (lane / 32) + e % 4.  The owners (queries in the forward and
// query-gradient kernels, keys in the key/value-gradient kernel) are the columns,
// the streamed rows the result rows, so that a softmax statistic is a lane's own
// sum and one exchange between the lane halves, and eight consecutive entries
// of a score tile are the B operand of the product that follows: contraction
// slot (half, j) stands for streamed row 16 s + 8 (j / 4) + 4 half + j % 4,
// and the A operand reads its rows in the same order (col_frag).
//
// Streamed rows go through two LDS buffers, by way of registers: one barrier a
// tile, the next tile's loads in flight during the products, rows past the
// sequence and elements past the head dimension set to zero on the way.
#pragma once
#include <type_traits>

#include "eql_attn_args.h"
#include "eql_common.h"
#include "eql_config.h"
#include "eql_gemm.h"

namespace eqk {

typedef float floatx16 __attribute__((ext_vector_type(16)));

// Bits as the other type.  By value: a bit cast of an element of a vector names
// the vector's first element in this compiler.
__device__ __forceinline__ float bits_f32(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t f32_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// Eight contraction values of one row: a lane's share of a 16-deep step.
template <int DT>
struct Frag8 {
  uint32_t w[DT == kF32 ? 8 : 4];
};

template <int DT>
__device__ __forceinline__ void mma32(floatx16& acc, const Frag8<DT>& a, const Frag8<DT>& b) {
  if constexpr (DT == kF16) {
    const u32x4 av = {a.w[0], a.w[1], a.w[2], a.w[3]}, bv = {b.w[0], b.w[1], b.w[2], b.w[3]};
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, av), __builtin_bit_cast(half8, bv), acc, 0,
                                                 0, 0);
  } else if constexpr (DT == kBF16) {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    const u32x4 av = {a.w[0], a.w[1], a.w[2], a.w[3]}, bv = {b.w[0], b.w[1], b.w[2], b.w[3]};
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av), __builtin_bit_cast(bf16x8, bv), acc,
                                                  0, 0, 0);
  } else {
    // step j of the eight contracts slot j of both lane halves
#pragma unroll
    for (int j = 0; j < 8; ++j)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, a.w[j]), __builtin_bit_cast(float, b.w[j]),
                                                 acc, 0, 0, 0);
  }
}

// Two floats rounded to nearest even and packed by one instruction.
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  using E = typename Elem<DT>::T;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef E e16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), e16x2));
}

// Entries 8 s .. 8 s + 7 of a result tile, rounded to the element type, as the
// operand of a 16-deep step.
template <int DT>
__device__ __forceinline__ Frag8<DT> tile_frag(const floatx16& t, int s) {
  Frag8<DT> f;
  if constexpr (DT == kF32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f.w[j] = f32_bits(t[8 * s + j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) f.w[j] = pack_pair<DT>(t[8 * s + 2 * j], t[8 * s + 2 * j + 1]);
  }
  return f;
}

// sum + the eight values of an operand, as rounded
template <int DT>
__device__ __forceinline__ float add_frag(float sum, const Frag8<DT>& f) {
  if constexpr (DT == kF32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += bits_f32(f.w[j]);
  } else if constexpr (DT == kF16) {
    const half2v one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = f.w[j];
      sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w), one, sum, false);
    }
  } else {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = f.w[j];
      sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), one, sum, false);
    }
  }
  return sum;
}

// LDS tile of rows of DP elements.  16-byte chunk c of a row lies at chunk
// c ^ swz(row): sixteen consecutive rows put one chunk on sixteen places of the 256
// bytes of all banks (row reads), and four consecutive rows put four
// neighbouring chunks on sixteen (transposed reads).
template <int DT, int DP>
struct RowTile {
  static constexpr int EB = DT == kF32 ? 4 : 2;
  static constexpr int CE = 16 / EB;                        // elements of a chunk
  static constexpr int NC = DP / CE;                        // chunks of a row
  static constexpr int RB = (DP == 96 ? 128 : DP) * EB;     // bytes of a row
  static constexpr int NCH = RB / 16;
  __device__ static __forceinline__ int swz(int row) {
    if constexpr (NCH == 4) return (row >> 2) & 3;
    else if constexpr (NCH == 8) return ((row >> 1) & 1) * 4 + ((row >> 2) & 3);
    else return (row & 3) * 4 + ((row >> 2) & 3);
  }
  __device__ static __forceinline__ int off(int row, int c) { return row * RB + ((c ^ swz(row)) << 4); }
};

// A lane's places in a tile.  16 bits: offsets formed once, to which a tile's
// place in LDS and a row block are compile-time constants of the instruction (rows
// 16 apart share their swizzle), a step or column block flips bits of the chunk.
template <int DT, int DP>
struct LdsMap {
  using RT = RowTile<DT, DP>;
  int lane, first;  // first tile row, a multiple of 32
  uint32_t row0, col0[2];
  __device__ __forceinline__ explicit LdsMap(int lane_, int first_ = 0) : lane(lane_), first(first_) {
    row0 = RT::off(first + (lane & 31), lane >> 5);
    const int e = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      col0[j] = RT::off(first + 8 * j + 4 * (lane >> 5) + ((lane & 15) >> 2), e / RT::CE) + e % RT::CE * RT::EB;
  }
  // The compiler forms the flipped offsets anew from here on instead of keeping them
  // all: a kernel short of registers calls it once a tile.
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(row0), "+v"(col0[0]), "+v"(col0[1])); }
  // Row operand: elements 16 s + 8 half .. + 7 of tile row 32 n + lane % 32.
  __device__ __forceinline__ Frag8<DT> row(const char* t, int n, int s) const {
    Frag8<DT> f;
    if constexpr (DT == kF32) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(t + RT::off(first + n * 32 + (lane & 31), (2 * s + (lane >> 5)) * 2 + q));
#pragma unroll
        for (int j = 0; j < 4; ++j) f.w[4 * q + j] = a[j];
      }
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4*>(t + n * 32 * RT::RB + (row0 ^ (s << 5)));
#pragma unroll
      for (int j = 0; j < 4; ++j) f.w[j] = a[j];
    }
    return f;
  }
  // Column operand: element 32 d + lane % 32 of tile rows r0 + 8 (j / 4) + 4 half + j % 4,
  // r0 a multiple of 16.  16 bits: two transposing LDS reads, in which sixteen lanes
  // hand in the addresses of four rows of sixteen elements and lane i takes column i.
  __device__ __forceinline__ Frag8<DT> col(const char* t, int r0, int d) const {
    Frag8<DT> f;
    if constexpr (DT == kF32) {
      const int e = d * 32 + (lane & 31);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = first + r0 + 8 * (j >> 2) + 4 * (lane >> 5) + (j & 3);
        f.w[j] = *reinterpret_cast<const uint32_t*>(t + RT::off(row, e >> 2) + (e & 3) * 4);
      }
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(t + r0 * RT::RB + (col0[j] ^ (d << 6))));
        const u32x2 w = __builtin_bit_cast(u32x2, v);
        f.w[2 * j] = w[0];
        f.w[2 * j + 1] = w[1];
      }
    }
    return f;
  }
};

// Maximum and sum of the two lane halves' values.
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
  return fmaxf(bits_f32(r[0]), bits_f32(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
  return bits_f32(r[0]) + bits_f32(r[1]);
}

// Visibility of 32 streamed rows as bits.  below(x): bits 0 .. x - 1.
__device__ __forceinline__ uint32_t below(int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u; }
// All ones where the lane's owner sees entry e of a result tile, else zero; `bits`
// shifted right by 4 for the upper lane half.
__device__ __forceinline__ uint32_t entry_mask(uint32_t bits, int e) {
  return (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (e >> 2) + (e & 3), 1);
}

// Running maximum of the exponent fields of 16-byte chunks: equal to the mask in
// some field iff an infinity or NaN went by.
template <int DT>
struct ExpMax {
  static constexpr uint32_t kMask = DT == kF32 ? 0x7f800000u : DT == kF16 ? 0x7c007c00u : 0x7f807f80u;
  uint32_t m = 0;
  __device__ __forceinline__ void add(const u32x4& c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t e = c[j] & kMask;
      if constexpr (DT == kF32) {
        m = m > e ? m : e;
      } else {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, e)));
      }
    }
  }
  __device__ __forceinline__ bool hit() const {
    if constexpr (DT == kF32) return m == kMask;
    else return (m & 0xffffu) == (kMask & 0xffffu) || (m >> 16) == (kMask >> 16);
  }
};

// One 16-deep step of a product whose streamed rows hold infinities or NaN, and
// of which some owners see only some: the finite elements as ever (an owner who
// sees none of the others gets the very same bits), then the others row by row, each
// into a tile of its own that only the owners who see the row add.  sees(k) tells
// whether the lane's owner sees tile row k.
template <int DT, int DP, typename F>
__device__ __forceinline__ void mma_seen(floatx16 (&acc)[DP / 32], const LdsMap<DT, DP>& map, const char* t, int r0,
                                         const Frag8<DT>& b, F&& sees) {
  constexpr int NR = DT == kF32 ? 8 : 4;
  constexpr uint32_t kMask = ExpMax<DT>::kMask;
  const int half = map.lane >> 5;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) {
    Frag8<DT> a = map.col(t, r0, d), odd;
    bool any = false;
#pragma unroll
    for (int w = 0; w < NR; ++w) {
      const uint32_t e = a.w[w] & kMask;
      uint32_t m;
      if constexpr (DT == kF32) m = e == kMask ? 0xffffffffu : 0u;
      else m = ((e & 0xffffu) == (kMask & 0xffffu) ? 0xffffu : 0u) | ((e >> 16) == (kMask >> 16) ? 0xffff0000u : 0u);
      odd.w[w] = a.w[w] & m;
      a.w[w] &= ~m;
      any |= m != 0;
    }
    mma32<DT>(acc[d], a, b);
    if (!__any(any)) continue;
#pragma unroll 1
    for (int slot = 0; slot < 16; ++slot) {
      const int j = slot & 7;
      const bool mine = (slot >> 3) == half;
      const uint32_t keep = DT == kF32 ? 0xffffffffu : (j & 1) ? 0xffff0000u : 0x0000ffffu;
      Frag8<DT> one;
#pragma unroll
      for (int w = 0; w < NR; ++w) one.w[w] = mine && w == (DT == kF32 ? j : j >> 1) ? odd.w[w] & keep : 0u;
      floatx16 p{};
      mma32<DT>(p, one, b);
      const bool s = sees(r0 + 8 * (j >> 2) + 4 * (slot >> 3) + (j & 3));
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] += s ? p[e] : 0.0f;
    }
  }
}

// Whether a wave of the workgroup found infinities or NaN in the tile; the same in
// every wave.  The kernels walk their tiles on the assumption that there are none where
// they would matter (a tile that some owner sees in part) and, where it fails,
// start over with mma_seen: the common loop then carries nothing for it.
template <int NW>
__device__ __forceinline__ bool any_flag(const int* flag) {
  int f = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) f |= flag[w];
  return __builtin_amdgcn_readfirstlane(f) != 0;
}

// Orders a wave's LDS writes before its reads by other lanes, and the other way round:
// the hardware runs them in order, the compiler has to keep them so.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Loads of one streamed tile of TK rows by NT threads, held in registers between
// the load and the LDS write.  Buffer loads: an offset past the resource
// (kDropOffset, or a row past its end) reads as zero, so a row needs no arithmetic
// but its offset, the same in every tile.
template <int DT, int DP, int TK, int NT>
struct Stage {
  using RT = RowTile<DT, DP>;
  static constexpr int N = TK * RT::NC / NT;
  static_assert(TK * RT::NC % NT == 0, "whole chunks");
  u32x4 r[N];
  uint32_t off[N];
  // at(row): byte offset of tile row `row`; elements from D on are zero
  template <typename A>
  __device__ __forceinline__ void place(int tid, int D, A&& at) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = tid + i * NT, c = u % RT::NC;
      off[i] = c * RT::CE < D ? (uint32_t)at(u / RT::NC) + c * 16 : kDropOffset;
    }
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off[i], 0, 0));
  }
  // the tile rows from `rows` on as zero, whatever their offset
  __device__ __forceinline__ void load_first(__amdgpu_buffer_rsrc_t rs, int tid, int rows) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      r[i] = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (tid + i * NT) / RT::NC < rows ? off[i] : kDropOffset, 0, 0));
  }
  __device__ __forceinline__ void store(int tid, char* t) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = tid + i * NT;
      *reinterpret_cast<u32x4*>(t + RT::off(u / RT::NC, u % RT::NC)) = r[i];
    }
  }
  __device__ __forceinline__ void scan(ExpMax<DT>& m) const {
#pragma unroll
    for (int i = 0; i < N; ++i) m.add(r[i]);
  }
};
// Rows k0 .. of one sequence's keys or values (`base`, `stride` bytes a row), those
// below len, as a resource for one tile.
template <int TK>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_rsrc(const char* base, int64_t stride, int k0, int len, int row_bytes) {
  return make_rsrc(base + k0 * stride, (uint32_t)((min(len - k0, TK) - 1) * (int)stride + row_bytes));
}

// Owner operand: one row of D elements read straight from memory, steps of 16.
template <int DT, int DP>
__device__ __forceinline__ void load_owner(Frag8<DT> (&f)[DP / 16], const char* row, bool ok, int D, int half) {
  constexpr int N = DT == kF32 ? 2 : 1, CE = RowTile<DT, DP>::CE;
#pragma unroll
  for (int s = 0; s < DP / 16; ++s)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int c = (2 * s + half) * N + n;
      u32x4 v{0, 0, 0, 0};
      if (ok && c * CE < D) v = *reinterpret_cast<const u32x4*>(row + c * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[s].w[4 * n + j] = v[j];
    }
}

// Writes an owner's row from result tiles acc[DP / 32] (entries in d), times
// `mul`, rounded once, or zeros where it has no data: whole 16-byte words after
// an exchange between the halves.  Every lane of the wave must come here.
template <int DT, int DP>
__device__ __forceinline__ void store_owner(const floatx16 (&acc)[DP / 32], float mul, bool data, char* row,
                                            bool ok, int D, int half) {
  auto val = [&](int d, int e) { return data ? acc[d][e] * mul : 0.0f; };
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) {
    if constexpr (DT == kF32) {
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int at = 32 * d + 2 * e + 4 * half;
        const floatx4 v = {val(d, e), val(d, e + 1), val(d, e + 2), val(d, e + 3)};
        if (ok && at < D) *reinterpret_cast<floatx4*>(row + at * 4) = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; e += 8) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_pair<DT>(val(d, e + 2 * j), val(d, e + 2 * j + 1));
        const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        const int at = 32 * d + 2 * e + 8 * half;
        if (ok && at < D) *reinterpret_cast<u32x4*>(row + at * 2) = u32x4{a[0], b[0], a[1], b[1]};
      }
    }
  }
}

// Length and start of one sequence, in the ranges the position arithmetic allows.
__device__ __forceinline__ int seq_len(const AttnArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.Lk) : a.Lk;
}
__device__ __forceinline__ int seq_start(const AttnArgs& a, int b) {
  return a.starts ? min(max(a.starts[b], -kAttnMaxPos), kAttnMaxPos) : a.Lk - a.Lq;
}

// The keys that packed rows r0 .. r1 see, as key tiles of TK: `ns` tiles of first
// tokens, then tiles t0 ...; n in all.  And per range the bounds of visibility.
struct KeyRange {
  int n, ns, t0;
  int last, sink_end;     // no row sees past `last`; first tokens seen by some row
  int first;              // no row sees before `first`, first tokens aside
  int all_first, all_last, all_sink;  // keys every row sees: all_first .. all_last and below all_sink
  __device__ __forceinline__ int tile(int i) const { return i < ns ? i : t0 + i - ns; }
  // whether every row sees the whole tile from key k0 on
  __device__ __forceinline__ bool whole(int k0, int TK) const {
    return k0 + TK - 1 <= all_last && (k0 >= all_first || k0 + TK <= all_sink);
  }
};
__device__ __forceinline__ KeyRange key_range(const AttnArgs& a, int r0, int r1, int len, int start, int TK) {
  KeyRange k{};
  const int pa = start + r0 / a.G, pb = min(start + r1 / a.G, len - 1);
  if (pa > pb) { k.last = -1; k.first = 1; return k; }
  k.last = min(len - 1, pb + a.right);
  k.first = max(0, pa - a.left);
  k.sink_end = min(a.sinks, k.last + 1);
  k.all_first = pb - a.left;
  k.all_last = min(len - 1, pa + a.right);
  k.all_sink = min(a.sinks, k.all_last + 1);
  if (k.last < 0) return k;
  k.t0 = k.first / TK;
  k.ns = min((k.sink_end + TK - 1) / TK, k.t0);
  k.n = k.ns + max(k.last / TK - k.t0 + 1, 0);
  return k;
}

// Workgroup number -> (sequence and key/value head, item of its n).  Workgroup i runs
// on XCD i % 8.  From 16 items on, every XCD takes two runs of n / 16 neighbouring
// items of each head pair, the k-th and the (15 - k)-th, k turning with the pair:
// neighbours share what they stream in one L2, and every XCD has its share of a ragged
// batch's long sequences and of work that grows along the sequence.  The runs of the
// half where the work is come first, of all head pairs, the others fill the end.
// Fewer items: one XCD takes whole head pairs.
struct Item {
  int bh, at;
  bool ok;
};
template <bool LATE>
__device__ __forceinline__ Item attn_item(uint32_t i, uint32_t blocks, uint32_t pairs, uint32_t n) {
  Item r;
  const uint32_t x = i % 8, s = i / 8;
  if (n < kAttnFold) {
    const uint32_t q = blocks / 8, rest = blocks % 8, id = x * q + min(x, rest) + s;
    r.bh = (int)(id / n);
    r.at = (int)(id % n);
    r.ok = true;
  } else {
    const uint32_t c = n / kAttnFold + 1;
    const bool second = s >= pairs * c;
    const uint32_t j = second ? s - pairs * c : s, in = j % c;
    r.bh = (int)(j / c);
    const uint32_t k = (x + r.bh) % 8, run = LATE != second ? 15 - k : k;
    const uint32_t lo = (uint32_t)((uint64_t)run * n / kAttnFold), hi = (uint32_t)((uint64_t)(run + 1) * n / kAttnFold);
    r.at = (int)(lo + in);
    r.ok = lo + in < hi;
  }
  return r;
}

// ---- forward ---------------------------------------------------------------
// o = sum_j p_j v_j / sum_j p_j, p_j = exp2(c s_j - m), c = scale log2 e, with the
// running maximum m of a row raised (and what was summed rescaled) only where
// a tile's maximum exceeds it by 2^8: probabilities stay below 2^8, far inside
// fp16's range.  Scores, maxima and sums in fp32; a probability is
// rounded once to the element type, as the operand of the second product.
// Two forms.  RW = 4 waves of 32 rows each share the staged tiles.  Up to 32 rows (new
// tokens over a cache): KEYS = 4 or 8 waves hold the same rows and take every KEYS-th tile
// each, in LDS of their own, without waiting for one another (a wave's LDS operations
// run in order, so one buffer does), and join at the end.
//
// Bound: heads of 64 by the vector pipe (130 instructions a wave and tile, 32 of them
// exponentials at a quarter rate, against 16 products of 32 cycles), wider ones by
// both pipes; few rows by memory.  16,389 tokens, 12 heads of 64, window +-1024, fp16:
// 157 us, 640 TFLOP/s (vector pipe 49% busy, products 30%, no LDS conflict, 2.1 waves a
// SIMD on average: the last of 6 workgroups a CU run alone).  One token over 16
// caches of up to 65,536 keys, 4 heads of 128, bf16: 240 us with the join, 5.5 TB/s.
template <int DT, int DP, int RW, int KEYS>
__global__ __launch_bounds__(RW * KEYS * 64, KEYS > 1 ? 2 : DT == kF32 ? 1 : DP > 64 ? 2 : 3) void eql_wattn_fwd_kernel(AttnArgs a) {
  using RT = RowTile<DT, DP>;
  static_assert(RW == 1 || KEYS == 1, "waves share rows or tiles");
  constexpr int TK = attn_fwd_tile(DT, RW), NBUF = RW == 1 ? 1 : 2, NT = RW * 64, NB = TK / 32, TB = TK * RT::RB;
  extern __shared__ __attribute__((aligned(16))) char smem_[];  // per key wave: K buffers, V buffers; flags or statistics
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave_ = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = RW == 1 ? 0 : wave_, kwave = KEYS == 1 ? 0 : wave_;
  const int tid = RW == 1 ? lane : threadIdx.x;  // among the threads that stage a tile
  char* const smem = smem_ + kwave * 2 * NBUF * TB;
  char* const tail = smem_ + KEYS * 2 * NBUF * TB;
  int* const flags = reinterpret_cast<int*>(tail);
  const int nrt = (a.R + 32 * RW - 1) / (32 * RW);
  const Item item = attn_item<true>(blockIdx.x, gridDim.x, (uint32_t)(a.B * a.Hkv), (uint32_t)nrt * a.parts);
  if (!item.ok) return;
  const int part = item.at % a.parts, rt = item.at / a.parts, bh = item.bh;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int len = seq_len(a, b), start = seq_start(a, b);

  const int g0 = rt * 32 * RW, g1 = min(g0 + 32 * RW, a.R) - 1;  // rows of the workgroup
  const int w0 = g0 + wave * 32, w1 = min(w0 + 31, a.R - 1);     // and of the wave
  const KeyRange kg = key_range(a, g0, g1, len, start, TK);
  KeyRange kw = key_range(a, w0, w1, len, start, TK);
  if (w0 > w1) { kw.n = 0; kw.last = -1; kw.first = 1; kw.sink_end = 0; }
  const int r = w0 + (lane & 31);
  const int tok = min(r, a.R - 1) / a.G, pos = start + tok;
  const int head = hk * a.G + min(r, a.R - 1) % a.G;
  const bool row_ok = r < a.R && pos < len;
  const int hi = row_ok ? min(len - 1, pos + a.right) : -1, lo = pos - a.left, sk = min(a.sinks, hi + 1);

  // bit k: whether the lane's row sees key k0 + k
  auto seen_bits = [&](int k0) { return below(hi - k0 + 1) & (~below(lo - k0) | below(sk - k0)); };
  const char* const kb = (const char*)a.k + ((int64_t)b * a.ks[0] + (int64_t)hk * a.ks[2]) * RT::EB;
  const char* const vb = (const char*)a.v + ((int64_t)b * a.vs[0] + (int64_t)hk * a.vs[2]) * RT::EB;
  Frag8<DT> qf[DP / 16];
  load_owner<DT, DP>(qf, (const char*)a.q + ((int64_t)b * a.qs[0] + (int64_t)tok * a.qs[1] + (int64_t)head * a.qs[2]) * RT::EB,
                     row_ok, a.D, half);

  const int i0 = (int)((int64_t)kg.n * part / a.parts), i1 = (int)((int64_t)kg.n * (part + 1) / a.parts);
  Stage<DT, DP, TK, NT> sk_, sv_;
  const int64_t kst = a.ks[1] * RT::EB, vst = a.vs[1] * RT::EB;
  sk_.place(tid, a.D, [&](int row) { return row * (int)kst; });
  sv_.place(tid, a.D, [&](int row) { return row * (int)vst; });
  auto load = [&](int i) {
    const int k0 = kg.tile(i) * TK;
    sk_.load(row_rsrc<TK>(kb, kst, k0, len, a.D * RT::EB));
    sv_.load(row_rsrc<TK>(vb, vst, k0, len, a.D * RT::EB));
  };

  floatx16 acc[DP / 32];
  float m, l;
  const float c = a.scale_log2e;
  const LdsMap<DT, DP> map(lane);
  auto walk = [&](auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) acc[d] = floatx16{};
    m = -__builtin_inff();
    l = 0.0f;
    if (i0 + kwave < i1) load(i0 + kwave);
    auto step = [&](int i, auto which) {
      constexpr int buf = decltype(which)::value;
      char* const kt = smem + buf * TB;
      char* const vt = smem + (NBUF + buf) * TB;
      int* const flag = flags + buf * RW;
      sk_.store(tid, kt);
      sv_.store(tid, vt);
      const int k0 = kg.tile(i) * TK;
      const bool part_seen = !kg.whole(k0, TK);  // some row sees the tile in part
      bool odd = false;
      if (part_seen) {
        ExpMax<DT> e;
        sv_.scan(e);
        odd = __any(e.hit());
        if (KEYS == 1 && lane == 0) flag[wave] = odd;
      }
      if constexpr (KEYS == 1) __syncthreads();
      else wave_lds_fence();
      if (i + KEYS < i1) load(i + KEYS);
      if constexpr (!kCareful) {
        if (part_seen && (KEYS == 1 ? any_flag<RW>(flag) : odd)) return false;
      }
      if (k0 > kw.last || (k0 + TK <= kw.first && k0 >= kw.sink_end)) return true;  // no row of the wave sees the tile
      floatx16 s[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        s[n] = floatx16{};
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) mma32<DT>(s[n], map.row(kt, n, t), qf[t]);
      }
      const bool whole = kw.whole(k0, TK);
      auto sees = [&](int k) { return bool((seen_bits(k0 + (k & 32)) >> (k & 31)) & 1u); };
      if (!whole) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const uint32_t bits = seen_bits(k0 + 32 * n) >> (4 * half);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t k = entry_mask(bits, e);
            s[n][e] = bits_f32((f32_bits(s[n][e]) & k) | (0xff800000u & ~k));  // -inf
          }
        }
      }
      float mx = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[n][e]);
      mx = half_max(mx);
      if (__any((mx - m) * c > 8.0f)) {
        const float mn = fmaxf(m, mx);
        const float f = mn == m ? 1.0f : __builtin_amdgcn_exp2f((m - mn) * c);
        m = mn;
        l *= f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] *= f;
      }
      const float mc = m == -__builtin_inff() ? 0.0f : m * c;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[n][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][e], c, -mc));
#pragma unroll
      for (int t = 0; t < 2 * NB; ++t) {
        const Frag8<DT> p = tile_frag<DT>(s[t / 2], t % 2);
        l = add_frag<DT>(l, p);  // of the rounded probabilities, as the numerator
        if constexpr (kCareful) {
          mma_seen<DT, DP>(acc, map, vt, 16 * t, p, sees);
        } else {
#pragma unroll
          for (int d = 0; d < DP / 32; ++d) mma32<DT>(acc[d], map.col(vt, 16 * t, d), p);
        }
      }
      return true;
    };
    for (int i = i0 + kwave; i < i1; i += NBUF * KEYS) {
      if (!step(i, std::integral_constant<int, 0>{})) return false;
      if constexpr (KEYS > 1) wave_lds_fence();
      if constexpr (NBUF == 2)
        if (i + 1 < i1 && !step(i + 1, std::integral_constant<int, 1>{})) return false;
    }
    return true;
  };
  if (!walk(std::false_type{})) {
    if constexpr (KEYS == 1) __syncthreads();
    walk(std::true_type{});
  }
  if constexpr (KEYS > 1) {
    // the waves' sums to the first wave, each through its own part of the LDS
    float* const x = reinterpret_cast<float*>(smem_) + lane;
    float2* const st = reinterpret_cast<float2*>(tail) + lane;
    constexpr int kWave = 2 * NBUF * TB / 4;
    wave_lds_fence();
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[kwave * kWave + (d * 16 + e) * 64] = acc[d][e];
    st[kwave * 64] = make_float2(m, l);
    __syncthreads();
    if (kwave != 0) return;
#pragma unroll
    for (int w = 1; w < KEYS; ++w) m = fmaxf(m, st[w * 64].x);
    l = 0.0f;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) acc[d] = floatx16{};
    for (int w = 0; w < KEYS; ++w) {
      const float2 v = st[w * 64];
      const float f = v.x == -__builtin_inff() ? 0.0f : v.x == m ? 1.0f : __builtin_amdgcn_exp2f((v.x - m) * c);
      l += v.y * f;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float y = x[w * kWave + (d * 16 + e) * 64];
          acc[d][e] += f == 0.0f ? 0.0f : y * f;  // a wave that saw nothing holds no numbers
        }
    }
  }
  l = half_sum(l);
  if (!row_ok) l = 0.0f;
  const float ml = m == -__builtin_inff() ? 0.0f : m * c;
  const int64_t row = (int64_t)bh * a.R + r;
  if (a.parts == 1) {
    store_owner<DT, DP>(acc, 1.0f / l, l != 0.0f,
                        (char*)a.o + ((int64_t)b * a.os[0] + (int64_t)tok * a.os[1] + (int64_t)head * a.os[2]) * RT::EB,
                        r < a.R, a.D, half);
    if (a.lse && half == 0 && r < a.R) a.lse[row] = l == 0.0f ? __builtin_inff() : ml + __builtin_amdgcn_logf(l);
  } else {
    // part of a row: the unscaled sums, then maximum and sum
    const int64_t rows = (int64_t)a.B * a.Hkv * a.R, at = (int64_t)part * rows + row;
    store_owner<kF32, DP>(acc, 1.0f, true, (char*)(a.part + at * a.D), r < a.R, a.D, half);
    if (half == 0 && r < a.R) {
      float* const st = a.part + rows * a.parts * a.D + at * 2;
      st[0] = l == 0.0f ? -__builtin_inff() : ml;
      st[1] = l;
    }
  }
}

// Joins the parts of each row (64 at most): lane p of a wave holds part p's statistics.
// Up to 8 parts a wave adds a row's parts in their order; more are dealt to the four
// waves of a workgroup, whose sums are added in theirs (32 parts of 1,024 rows of 128
// one after another 18 us).
template <int DT>
__global__ __launch_bounds__(256) void eql_wattn_join_kernel(AttnArgs a) {
  using E = typename Elem<DT>::T;
  __shared__ float add[4][2][64];
  const int64_t rows = (int64_t)a.B * a.Hkv * a.R;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int deal = attn_join_waves(a.parts), first = deal == 1 ? 0 : wave;
  const int64_t row = deal == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= rows) return;  // only where a wave has a row of its own
  float m = -__builtin_inff(), l = 0.0f;
  if (lane < a.parts) {
    const float2 v = ((const float2*)(a.part + rows * a.parts * a.D))[(int64_t)lane * rows + row];
    m = v.x;
    l = v.y;
  }
  float top = m;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  const float mu = top == -__builtin_inff() ? 0.0f : top;
  const float f = __builtin_amdgcn_exp2f(m - mu);
  l = l == 0.0f ? 0.0f : l * f;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
  float o0 = 0.0f, o1 = 0.0f;
  const bool c0 = lane < a.D, c1 = lane + 64 < a.D;
#pragma unroll 8
  for (int p = first; p < a.parts; p += deal) {
    const float* const x = a.part + (p * rows + row) * a.D + lane;
    const float g = __shfl(f, p);
    const float x0 = c0 ? x[0] : 0.0f, x1 = c1 ? x[64] : 0.0f;
    o0 += g == 0.0f ? 0.0f : x0 * g;  // a part that saw nothing holds no numbers
    o1 += g == 0.0f ? 0.0f : x1 * g;
  }
  if (deal > 1) {
    add[wave][0][lane] = o0;
    add[wave][1][lane] = o1;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < 4; ++w) {
      o0 += add[w][0][lane];
      o1 += add[w][1][lane];
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int bh = (int)(row / a.R), r = (int)(row % a.R);
  E* const o = (E*)a.o + ((int64_t)(bh / a.Hkv) * a.os[0] + (int64_t)(r / a.G) * a.os[1] +
                          (int64_t)((bh % a.Hkv) * a.G + r % a.G) * a.os[2]);
  if (c0) o[lane] = (E)(o0 * inv);
  if (c1) o[lane + 64] = (E)(o1 * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? __builtin_inff() : mu + __builtin_amdgcn_logf(l);
}

// fp16: score gradients are rounded as the operand of a product times a power of two of
// their owner (a query's row, a key's column), so that neither large values overflow fp16's
// range nor small gradients fall below it.  The power starts where a product of fp16's two smallest
// numbers counts, and comes down as a running maximum goes up: where a tile holds an entry
// of more than 2^15, the owner's largest is taken to about 2^kRaised, and what was summed with it.
// An entry 2^17 times smaller than its owner's largest keeps all its bits.  Infinities stay.
// The maximum costs up to 5% of a gradient (16,389 tokens, 12 heads of 64, window +-1024: 495 -> 508 us).
constexpr float kRaiseStart = 0x1p60f, kRaiseLimit = 0x1p15f;
constexpr int kRaised = 4;
template <int DP>
__device__ __forceinline__ void lower_raise(floatx16& t, floatx16 (&acc)[DP / 32], float& up) {
  float mx = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) mx = fmaxf(mx, __builtin_fabsf(t[e]));
  if (!__any(mx > kRaiseLimit)) return;
  mx = half_max(mx);
  const int low = mx > kRaiseLimit && mx < __builtin_inff() ? __builtin_amdgcn_frexp_expf(mx) - kRaised : 0;
  const float f = __builtin_ldexpf(1.0f, -low);
  up *= f;
#pragma unroll
  for (int e = 0; e < 16; ++e) t[e] *= f;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] *= f;
}

// ---- query gradient --------------------------------------------------------
// dq = scale sum_j ds_j k_j, ds_j = p_j (do . v_j - delta), p_j = exp2(c s_j - lse),
// delta = do . o = sum_j p_j do . v_j, which it writes for the kernel that follows.  16 bits: the
// rounded o would put an error of u |do| |o| into a difference of numbers that are larger by
// sqrt(keys) only, so a workgroup with a row that sees at most kFewKeys keys first walks its tiles for
// sum_j p_j do . v_j over sum_j p_j (dq and dk of rows of two keys 1.5 times as far from the exact
// ones as results rounded once, from the rounded o 2.2; of five keys 1.45 and 1.7; from 33 keys on
// it makes 0.1 of a difference).  Elsewhere do . o of the rounded o; ds rounded costs 1.4 by itself.
// Windows of 16 keys over 4,096 tokens run as fast either way, both gradients 104 - 110 us.
//
// Three products where the forward has two, and bound like it.  2 ragged clips of up to
// 8,197 tokens, 16 heads of 128 on 4, window 2047, bf16: 300 - 330 us.
constexpr int kFewKeys = 32;
template <int DT, int DP, int NW>
__global__ __launch_bounds__(NW * 64, DT == kF32 ? 1 : 2) void eql_wattn_dq_kernel(AttnArgs a) {
  using RT = RowTile<DT, DP>;
  constexpr int TK = attn_tile(DT), NBUF = 2, NT = NW * 64, NB = TK / 32, TB = TK * RT::RB;
  extern __shared__ __attribute__((aligned(16))) char smem[];  // K 0, K 1, V 0, V 1, flags
  int* const flags = reinterpret_cast<int*>(smem + 4 * TB);
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item item = attn_item<true>(blockIdx.x, gridDim.x, (uint32_t)(a.B * a.Hkv), (uint32_t)((a.R + 32 * NW - 1) / (32 * NW)));
  if (!item.ok) return;
  const int rt = item.at, bh = item.bh;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int len = seq_len(a, b), start = seq_start(a, b);
  const int g0 = rt * 32 * NW, g1 = min(g0 + 32 * NW, a.R) - 1;
  const int w0 = g0 + wave * 32, w1 = min(w0 + 31, a.R - 1);
  const KeyRange kg = key_range(a, g0, g1, len, start, TK);
  KeyRange kw = key_range(a, w0, w1, len, start, TK);
  if (w0 > w1) { kw.n = 0; kw.last = -1; kw.first = 1; kw.sink_end = 0; }
  const int r = w0 + (lane & 31);
  const int tok = min(r, a.R - 1) / a.G, pos = start + tok;
  const int head = hk * a.G + min(r, a.R - 1) % a.G;
  const bool row_ok = r < a.R && pos < len;
  const int hi = row_ok ? min(len - 1, pos + a.right) : -1, lo = pos - a.left, sk = min(a.sinks, hi + 1);
  auto at = [&](const void* p, const int64_t (&s)[3]) {
    return (char*)p + ((int64_t)b * s[0] + (int64_t)tok * s[1] + (int64_t)head * s[2]) * RT::EB;
  };
  // bit k: whether the lane's row sees key k0 + k
  auto seen_bits = [&](int k0) { return below(hi - k0 + 1) & (~below(lo - k0) | below(sk - k0)); };
  const char* const kb = (const char*)a.k + ((int64_t)b * a.ks[0] + (int64_t)hk * a.ks[2]) * RT::EB;
  const char* const vb = (const char*)a.v + ((int64_t)b * a.vs[0] + (int64_t)hk * a.vs[2]) * RT::EB;
  const int64_t row = (int64_t)bh * a.R + r;
  const float lse = row_ok ? a.lse[row] : __builtin_inff();
  // whether some row of the workgroup sees few keys (the first and last see the fewest)
  auto keys_of = [&](int p) {
    const int last = min(len - 1, p + a.right), first = max(0, p - a.left);
    return max(last - first + 1, 0) + min(a.sinks, min(first, last + 1));
  };
  const bool few = DT != kF32 && kg.n > 0 && min(keys_of(start + g0 / a.G), keys_of(min(start + g1 / a.G, len - 1))) <= kFewKeys;
  float delta = 0.0f;
  if (row_ok && !few) {
    // each half of the wave takes every second chunk of the row
    const char *const po = at(a.o, a.os), *const pg = at(a.go, a.gos);
#pragma unroll 1
    for (int e = half * RT::CE; e < a.D; e += 2 * RT::CE) {
      const u32x4 vo = *reinterpret_cast<const u32x4*>(po + e * RT::EB), vg = *reinterpret_cast<const u32x4*>(pg + e * RT::EB);
      const uint32_t wo[4] = {vo[0], vo[1], vo[2], vo[3]}, wg[4] = {vg[0], vg[1], vg[2], vg[3]};
      float x[RT::CE], y[RT::CE];
      raw_to_floats<DT, 4>(wo, x);
      raw_to_floats<DT, 4>(wg, y);
#pragma unroll
      for (int j = 0; j < RT::CE; ++j) delta = __builtin_fmaf(x[j], y[j], delta);
    }
  }
  delta = half_sum(delta);
  Frag8<DT> qf[DP / 16], gf[DP / 16];
  load_owner<DT, DP>(qf, at(a.q, a.qs), row_ok, a.D, half);
  load_owner<DT, DP>(gf, at(a.go, a.gos), row_ok, a.D, half);

  Stage<DT, DP, TK, NT> sk_, sv_;
  const int64_t kst = a.ks[1] * RT::EB, vst = a.vs[1] * RT::EB;
  sk_.place(tid, a.D, [&](int row) { return row * (int)kst; });
  sv_.place(tid, a.D, [&](int row) { return row * (int)vst; });
  auto load = [&](int i) {
    const int k0 = kg.tile(i) * TK;
    sk_.load(row_rsrc<TK>(kb, kst, k0, len, a.D * RT::EB));
    sv_.load(row_rsrc<TK>(vb, vst, k0, len, a.D * RT::EB));
  };
  floatx16 acc[DP / 32];
  float up;            // the power of two that ds is formed times
  float sum_p, sum_g;  // of a row's probabilities, and times do . v
  const float c = a.scale_log2e;
  const LdsMap<DT, DP> map(lane);
  auto walk = [&](auto mode) {
    constexpr bool kCareful = decltype(mode)::value == 1, kDelta = decltype(mode)::value == 2;
    sum_p = sum_g = 0.0f;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) acc[d] = floatx16{};
    up = DT == kF16 ? kRaiseStart : 1.0f;
    if (kg.n > 0) load(0);
    auto step = [&](int i, auto which) {
      constexpr int buf = decltype(which)::value;
      char* const kt = smem + buf * TB;
      char* const vt = smem + (2 + buf) * TB;
      int* const flag = flags + buf * NW;
      sk_.store(tid, kt);
      sv_.store(tid, vt);
      const int k0 = kg.tile(i) * TK;
      const bool part_seen = !kg.whole(k0, TK);  // some row sees the tile in part
      if (part_seen && !kDelta) {
        ExpMax<DT> e;
        sk_.scan(e);
        const bool any = __any(e.hit());
        if (lane == 0) flag[wave] = any;
      }
      __syncthreads();
      if (i + 1 < kg.n) load(i + 1);
      if constexpr (!kCareful && !kDelta) {
        if (part_seen && any_flag<NW>(flag)) return false;
      }
      if (k0 > kw.last || (k0 + TK <= kw.first && k0 >= kw.sink_end)) return true;
      const bool whole = kw.whole(k0, TK);
      auto sees = [&](int k) { return bool((seen_bits(k0 + (k & 32)) >> (k & 31)) & 1u); };
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        // a half of the tile that no row of the wave sees
        if (NB > 1 && (k0 + 32 * n > kw.last || (k0 + 32 * n + 32 <= kw.first && k0 + 32 * n >= kw.sink_end))) continue;
        floatx16 s{}, g{};
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
          mma32<DT>(s, map.row(kt, n, t), qf[t]);
          mma32<DT>(g, map.row(vt, n, t), gf[t]);
        }
        if constexpr (kDelta) {
          const uint32_t bits = whole ? ~0u : seen_bits(k0 + 32 * n) >> (4 * half);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -lse));
            sum_p += bits_f32(f32_bits(p) & entry_mask(bits, e));
            sum_g += bits_f32(f32_bits(p * g[e]) & entry_mask(bits, e));
          }
          continue;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -lse));
          s[e] = p * (DT == kF16 ? __builtin_fmaf(g[e], up, -delta * up) : g[e] - delta);
        }
        if (!whole) {
          const uint32_t bits = seen_bits(k0 + 32 * n) >> (4 * half);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = bits_f32(f32_bits(s[e]) & entry_mask(bits, e));
        }
        if constexpr (DT == kF16) lower_raise<DP>(s, acc, up);
        if constexpr (kCareful) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
            mma_seen<DT, DP>(acc, map, kt, n * 32 + 16 * t, tile_frag<DT>(s, t), sees);
        } else {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const Frag8<DT> p = tile_frag<DT>(s, t);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) mma32<DT>(acc[d], map.col(kt, n * 32 + 16 * t, d), p);
          }
        }
      }
      return true;
    };
    for (int i = 0; i < kg.n; i += NBUF) {
      if (!step(i, std::integral_constant<int, 0>{})) return false;
      if constexpr (NBUF == 2)
        if (i + 1 < kg.n && !step(i + 1, std::integral_constant<int, 1>{})) return false;
    }
    return true;
  };
  if (few) {
    walk(std::integral_constant<int, 2>{});
    sum_p = half_sum(sum_p);
    sum_g = half_sum(sum_g);
    delta = row_ok && sum_p != 0.0f ? sum_g / sum_p : 0.0f;
    __syncthreads();
  }
  if (half == 0 && r < a.R) a.delta[row] = delta;
  if (!walk(std::integral_constant<int, 0>{})) {
    __syncthreads();
    walk(std::integral_constant<int, 1>{});
  }
  store_owner<DT, DP>(acc, DT == kF16 ? a.scale / up : a.scale, row_ok, at(a.dq, a.dqs), r < a.R, a.D, half);
}

// ---- key and value gradient ------------------------------------------------
// dv_j = sum_r p_rj do_r, dk_j = scale sum_r ds_rj q_r over the packed rows r, a
// contiguous run for each key.  A wave owns 32 keys; key tiles that hold first tokens
// (seen by every later row) and tiles of long runs are split into parts along the rows,
// whose fp32 sums a second kernel adds in order.  fp16: p is rounded times 2^10 (the
// probabilities of a row of 100,000 keys would lie below its normal range).
//
// Bound: heads of 128 by waiting (1.3 waves a SIMD; products 25% busy, LDS 30%): a key
// tile streams the rows that see it, 4.4 MB for a window of 2047 over 4 heads, and 58%
// of that comes from the L2.  The clips above: 570 - 610 us (dk and dv in workgroups of their
// own, which stream twice as much: 1145); of full length both gradients 1.14 ms, in fp16, which
// spills more, 1.37.  64 x 197 tokens, 12 heads of 64, fp16: 48 us.

// Wave groups of a workgroup, each taking its share of every tile's rows for the same
// keys.  Heads of more than 96 16-bit elements take two: their accumulators leave no
// room for a second workgroup on a CU, and one wave a SIMD waits for each of its reads.
constexpr int dkv_groups(int DT, int DP) { return DT != kF32 && DP > 96 ? 2 : 1; }

template <int DT, int DP>
__global__ __launch_bounds__(256 * dkv_groups(DT, DP), DT == kF32 || DP == 96 ? 1 : 2) void eql_wattn_dkv_kernel(AttnArgs a) {
  using RT = RowTile<DT, DP>;
  constexpr int TQ = attn_tile(DT), NBUF = 2, GR = dkv_groups(DT, DP), NW = 4 * GR, NT = NW * 64, NB = TQ / 32 / GR, TB = TQ * RT::RB;
  extern __shared__ __attribute__((aligned(16))) char smem[];  // Q 0, Q 1, dO 0, dO 1, lse 0 1, delta 0 1, flags, V
  float* const stats = reinterpret_cast<float*>(smem + 4 * TB);
  int* const flags = reinterpret_cast<int*>(stats + 4 * TQ);
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave / 4, g32 = group * 32 * NB;  // first tile row of the wave
  // items of one head pair: sink tiles in sink_parts parts, then the others in key_parts
  const Item item = attn_item<false>(blockIdx.x, gridDim.x, (uint32_t)(a.B * a.Hkv),
                                     (uint32_t)(a.sink_tiles * a.sink_parts + (a.key_tiles - a.sink_tiles) * a.key_parts));
  if (!item.ok) return;
  const int bh = item.bh;
  int w = item.at, kt_, part, parts;
  if (w < a.sink_tiles * a.sink_parts) {
    parts = a.sink_parts;
    kt_ = w / parts;
    part = w % parts;
  } else {
    parts = a.key_parts;
    kt_ = a.sink_tiles + (w - a.sink_tiles * a.sink_parts) / parts;
    part = (w - a.sink_tiles * a.sink_parts) % parts;
  }
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int len = seq_len(a, b), start = seq_start(a, b);
  const int ends = min(len - 1 - start, a.Lq - 1);  // last token with data
  // tokens that see some key of ja .. jb, and tokens that see all of them
  auto tokens = [&](int ja, int jb, int& t0, int& t1, int& all0, int& all1) {
    t0 = min(max(ja - a.right - start, 0), a.Lq);
    t1 = ja < len ? ja < a.sinks ? ends : min(ends, jb + a.left - start) : -1;
    all0 = min(max(jb - a.right - start, 0), a.Lq);
    all1 = jb < len ? jb < a.sinks ? ends : min(ends, ja + a.left - start) : -1;
  };
  const int j0 = kt_ * kAttnDkvKeys, jw = j0 + wave % 4 * 32, j = jw + (lane & 31);
  int g0, g1, w0, w1, f0, f1, l0, l1, u0, u1;
  tokens(j0, j0 + kAttnDkvKeys - 1, g0, g1, u0, u1);
  const int all_lo = u0 * a.G, all_hi = u1 < u0 ? -1 : u1 * a.G + a.G - 1;  // rows that see every key of the workgroup
  tokens(jw, jw + 31, w0, w1, f0, f1);
  tokens(j, j, l0, l1, u0, u1);
  const int rlo = l0 * a.G, rhi = l1 < l0 ? -1 : l1 * a.G + a.G - 1;  // rows that see the lane's key
  // bit k: whether row r0 + k sees the lane's key
  auto seen_bits = [&](int r0) { return below(rhi - r0 + 1) & ~below(rlo - r0); };
  const int wlo = w0 * a.G, whi = w1 < w0 ? -1 : w1 * a.G + a.G - 1;
  const int flo = f0 * a.G, fhi = f1 < f0 ? -1 : f1 * a.G + a.G - 1;

  // the owners' operands: keys in registers, values too or, with two wave groups, in LDS
  Frag8<DT> kf[DP / 16], vf[GR == 2 ? 1 : DP / 16];
  char* const vt = reinterpret_cast<char*>(flags + 2 * NW);
  uint32_t v0 = 0;  // the lane's first value chunk there
  {
    const int jc = min(j, len - 1);
    load_owner<DT, DP>(kf, (const char*)a.k + ((int64_t)b * a.ks[0] + (int64_t)jc * a.ks[1] + (int64_t)hk * a.ks[2]) * RT::EB,
                       j < len, a.D, half);
    const char* const vrow = (const char*)a.v + ((int64_t)b * a.vs[0] + (int64_t)jc * a.vs[1] + (int64_t)hk * a.vs[2]) * RT::EB;
    if constexpr (GR == 1) {
      load_owner<DT, DP>(vf, vrow, j < len, a.D, half);
    } else {
      Frag8<DT> f[DP / 16];
      load_owner<DT, DP>(f, vrow, j < len, a.D, half);
      v0 = RT::off(j - j0, half);
#pragma unroll
      for (int t = 0; t < DP / 16; ++t)
        if (group == 0) *reinterpret_cast<u32x4*>(vt + (v0 ^ (t << 5))) = u32x4{f[t].w[0], f[t].w[1], f[t].w[2], f[t].w[3]};
    }
  }
  auto values = [&](int t) {
    if constexpr (GR == 1) {
      return vf[t];
    } else {
      Frag8<DT> f;
      const u32x4 x = *reinterpret_cast<const u32x4*>(vt + (v0 ^ (t << 5)));
#pragma unroll
      for (int k = 0; k < 4; ++k) f.w[k] = x[k];
      return f;
    }
  };
  const int tq0 = g0 * a.G / TQ, nt = g1 < g0 ? 0 : (g1 * a.G + a.G - 1) / TQ - tq0 + 1;
  const int i0 = (int)((int64_t)nt * part / parts), i1 = (int)((int64_t)nt * (part + 1) / parts);
  const int rend = max(ends + 1, 0) * a.G;  // rows with data
  const char* const qb = (const char*)a.q + ((int64_t)b * a.qs[0] + (int64_t)hk * a.G * a.qs[2]) * RT::EB;
  const char* const gb = (const char*)a.go + ((int64_t)b * a.gos[0] + (int64_t)hk * a.G * a.gos[2]) * RT::EB;
  Stage<DT, DP, TQ, NT> sq, sg;
  float st_lse = 0.0f, st_delta = 0.0f;
  // offsets of a tile's rows from its first token; the same in every tile where the
  // head group divides the tile
  auto place = [&](int first) {
    auto at = [&](const int64_t (&s)[3], int rr) {
      const unsigned x = (unsigned)(first + rr), t = x / (unsigned)a.G;
      return (int)t * (int)(s[1] * RT::EB) + (int)(x - t * a.G) * (int)(s[2] * RT::EB);
    };
    sq.place(tid, a.D, [&](int rr) { return at(a.qs, rr); });
    sg.place(tid, a.D, [&](int rr) { return at(a.gos, rr); });
  };
  const bool even = TQ % a.G == 0;
  place(0);
  const float inv_c = 1.0f / a.scale_log2e;
  constexpr float kRaiseP = DT == kF16 ? 10.0f : 0.0f;
  // 16 bits: the score product starts from -lse / c of its row, and p = exp2(c s).  Full precision: p =
  // exp2(c s - lse), formed at the end; a sum that starts at 10 or 100 loses the last bits of
  // scores of about one in each of its steps (errors of dk and dv 2 - 3 times the plain form's).
  constexpr bool kLseFirst = DT != kF32;
  // The tiles in a rotated order: workgroups whose runs overlap come to a tile at about
  // the same time, tile numbers equal modulo the length of a run, and find it in their
  // XCD's L2.  From the run's start on, 64 runs of one head pair side by side touch
  // 64 places, more than the L2 holds.
  const int turn = i1 > i0 ? (int)((unsigned)(2 * a.run_tiles - (tq0 + i0) % a.run_tiles) % (unsigned)(i1 - i0)) : 0;
  auto tile_of = [&](int i) {
    const int x = i + turn;
    return x < i1 ? x : x - (i1 - i0);
  };
  auto load = [&](int i) {
    const int r0 = (tq0 + tile_of(i)) * TQ, t0 = r0 / a.G;
    if (!even) place(r0 - t0 * a.G);
    const auto rq = make_rsrc(qb + t0 * a.qs[1] * RT::EB, 0x7fffffffu), rg = make_rsrc(gb + t0 * a.gos[1] * RT::EB, 0x7fffffffu);
    sq.load_first(rq, tid, rend - r0);
    sg.load_first(rg, tid, rend - r0);
    if (tid < TQ) {
      const bool ok = r0 + tid < rend;
      const int64_t at = (int64_t)bh * a.R + (ok ? r0 + tid : rend - 1);
      st_lse = ok ? (kRaiseP - a.lse[at]) * (kLseFirst ? inv_c : 1.0f) : -__builtin_inff();
      st_delta = ok ? -a.delta[at] : 0.0f;
    }
  };
  floatx16 dk[DP / 32], dv[DP / 32];
  float up;  // the power of two that ds is formed times, over that of p
  const float c = a.scale_log2e;
  // (the gradients' products start from -delta of their rows: ds = p g)
  LdsMap<DT, DP> map(lane, g32);
  auto walk = [&](auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      dk[d] = floatx16{};
      dv[d] = floatx16{};
    }
    up = DT == kF16 ? kRaiseStart * 0x1p-10f : 1.0f;
    if (i0 < i1) load(i0);
    auto step = [&](int i, auto which) {
      constexpr int buf = decltype(which)::value;
      char* const qt = smem + buf * TB;
      char* const gt = smem + (2 + buf) * TB;
      float* const ls = stats + buf * TQ;
      float* const de = stats + (2 + buf) * TQ;
      int* const flag = flags + buf * NW;
      sq.store(tid, qt);
      sg.store(tid, gt);
      if (tid < TQ) {
        ls[tid] = st_lse;
        de[tid] = st_delta;
      }
      const int r0 = (tq0 + tile_of(i)) * TQ;
      const bool part_seen = !(r0 >= all_lo && r0 + TQ - 1 <= all_hi);  // some key is seen by a part of the tile
      if (part_seen) {
        ExpMax<DT> e;
        sq.scan(e);
        sg.scan(e);
        const bool any = __any(e.hit());
        if (lane == 0) flag[wave] = any;
      }
      __syncthreads();
      if (i + 1 < i1) load(i + 1);
      if constexpr (!kCareful) {
        if (part_seen && any_flag<NW>(flag)) return false;
      }
      if (r0 > whi || r0 + TQ <= wlo) return true;
      if constexpr (GR == 2) {
        map.renew();
        asm volatile("" : "+v"(v0));
      }
      const bool whole = r0 >= flo && r0 + TQ - 1 <= fhi;
      auto sees = [&](int k) { return bool((seen_bits(r0 + g32 + (k & 32)) >> (k & 31)) & 1u); };
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if (NB > 1 && (r0 + 32 * n > whi || r0 + 32 * n + 32 <= wlo)) continue;  // no key of the wave is seen by these rows
        floatx16 s, g;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const floatx4 le = *reinterpret_cast<const floatx4*>(ls + g32 + n * 32 + 8 * x + 4 * half);
          const floatx4 dl = *reinterpret_cast<const floatx4*>(de + g32 + n * 32 + 8 * x + 4 * half);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            s[4 * x + y] = kLseFirst ? le[y] : 0.0f;
            g[4 * x + y] = dl[y];
          }
        }
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
          mma32<DT>(s, map.row(qt, n, t), kf[t]);
          mma32<DT>(g, map.row(gt, n, t), values(t));
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if constexpr (kLseFirst) s[e] = __builtin_amdgcn_exp2f(s[e] * c);
          else s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, ls[g32 + n * 32 + 8 * (e >> 2) + 4 * half + (e & 3)]));
          g[e] *= DT == kF16 ? s[e] * up : s[e];
        }
        if (!whole) {
          const uint32_t bits = seen_bits(r0 + g32 + 32 * n) >> (4 * half);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t k = entry_mask(bits, e);
            s[e] = bits_f32(f32_bits(s[e]) & k);
            g[e] = bits_f32(f32_bits(g[e]) & k);
          }
        }
        if constexpr (DT == kF16) lower_raise<DP>(g, dk, up);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          Frag8<DT> p, ds;
          p = tile_frag<DT>(s, t);
          ds = tile_frag<DT>(g, t);
          if constexpr (kCareful) {
            mma_seen<DT, DP>(dv, map, gt, n * 32 + 16 * t, p, sees);
            mma_seen<DT, DP>(dk, map, qt, n * 32 + 16 * t, ds, sees);
          } else {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
              mma32<DT>(dv[d], map.col(gt, n * 32 + 16 * t, d), p);
              mma32<DT>(dk[d], map.col(qt, n * 32 + 16 * t, d), ds);
            }
          }
        }
      }
      return true;
    };
    for (int i = i0; i < i1; i += NBUF) {
      if (!step(i, std::integral_constant<int, 0>{})) return false;
      if constexpr (NBUF == 2)
        if (i + 1 < i1 && !step(i + 1, std::integral_constant<int, 1>{})) return false;
    }
    return true;
  };
  if (!walk(std::false_type{})) {
    __syncthreads();
    walk(std::true_type{});
  }
  const float scale_k = DT == kF16 ? a.scale * 0x1p-10f / up : a.scale, mul_v = DT == kF16 ? 0x1p-10f : 1.0f;
  constexpr bool kScaleFirst = GR == 2 && DT == kF16;  // a key's two groups have powers of their own
  const float mul_k = kScaleFirst ? 1.0f : scale_k;
  if constexpr (GR == 2) {
    if constexpr (kScaleFirst) {
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[d][e] *= scale_k;
    }
    // the second group's sums to the first, one gradient after the other
    float* const x = reinterpret_cast<float*>(smem) + (wave % 4 * (DP / 2)) * 64 + lane;
    auto join = [&](floatx16 (&acc)[DP / 32]) {
      __syncthreads();
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (group == 1) x[(d * 16 + e) * 64] = acc[d][e];
      __syncthreads();
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (group == 0) acc[d][e] += x[(d * 16 + e) * 64];
    };
    join(dk);
    join(dv);
    if (group == 1) return;
  }
  if (parts == 1) {
    const bool ok = j < a.Lk;
    store_owner<DT, DP>(dk, mul_k, j < len, (char*)a.dk + ((int64_t)b * a.dks[0] + (int64_t)j * a.dks[1] + (int64_t)hk * a.dks[2]) * RT::EB,
                          ok, a.D, half);
    store_owner<DT, DP>(dv, mul_v, j < len, (char*)a.dv + ((int64_t)b * a.dvs[0] + (int64_t)j * a.dvs[1] + (int64_t)hk * a.dvs[2]) * RT::EB,
                          ok, a.D, half);
  } else {
    // slot of this workgroup among the split ones of its head pair: [slot][dk, dv][key][D]
    const int64_t slots = (int64_t)a.sink_tiles * (a.sink_parts > 1 ? a.sink_parts : 0) +
                          (int64_t)(a.key_tiles - a.sink_tiles) * (a.key_parts > 1 ? a.key_parts : 0);
    const int slot = a.sink_parts > 1 ? w : w - a.sink_tiles;
    float* const p = a.part + ((bh * slots + slot) * 2 * kAttnDkvKeys + (j - j0)) * a.D;
    store_owner<kF32, DP>(dk, mul_k, j < len, (char*)p, true, a.D, half);
    store_owner<kF32, DP>(dv, mul_v, j < len, (char*)(p + (int64_t)kAttnDkvKeys * a.D), true, a.D, half);
  }
}

// Adds the parts of split key tiles in their order: a thread four elements of one
// tile's gradient.
template <int DT>
__global__ __launch_bounds__(256) void eql_wattn_dkv_sum_kernel(AttnArgs a, int keys) {
  using E = typename Elem<DT>::T;
  const int split_sinks = a.sink_parts > 1 ? a.sink_tiles : 0;
  const int split_keys = a.key_parts > 1 ? a.key_tiles - a.sink_tiles : 0;
  const int per = split_sinks + split_keys;
  const uint32_t chunks = (uint32_t)(keys * a.D + 1023) / 1024;
  const uint32_t id = blockIdx.x / chunks;
  const int which = id % 2;
  const int x = (int)((id / 2) % per), bh = (int)((id / 2) / per);
  const int64_t slots = (int64_t)split_sinks * a.sink_parts + (int64_t)split_keys * a.key_parts;
  int tile, parts;
  int64_t slot;
  if (x < split_sinks) {
    tile = x;
    parts = a.sink_parts;
    slot = (int64_t)x * parts;
  } else {
    tile = a.sink_tiles + x - split_sinks;
    parts = a.key_parts;
    slot = (int64_t)split_sinks * a.sink_parts + (int64_t)(x - split_sinks) * parts;
  }
  const int i = (int)(blockIdx.x % chunks) * 1024 + threadIdx.x * 4;  // D is a multiple of 4
  if (i >= min(keys, a.Lk - tile * keys) * a.D) return;
  const int b = bh / a.Hkv, hk = bh % a.Hkv;
  const int64_t one = (int64_t)2 * keys * a.D;
  const float* const src = a.part + (bh * slots + slot) * one + (int64_t)which * keys * a.D + i;
  floatx4 s = *reinterpret_cast<const floatx4*>(src);
#pragma unroll 8
  for (int p = 1; p < parts; ++p) s += *reinterpret_cast<const floatx4*>(src + p * one);
  const int64_t* const st = which ? a.dvs : a.dks;
  E* const dst = (E*)(which ? a.dv : a.dk) + (int64_t)b * st[0] + (int64_t)hk * st[2] +
                 (int64_t)(tile * keys + i / a.D) * st[1] + i % a.D;
#pragma unroll
  for (int k = 0; k < 4; ++k) dst[k] = (E)s[k];
}

}  // namespace eqk
