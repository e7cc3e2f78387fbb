// eql_attn_args.h -- arguments and launch plan of the windowed attention kernels,
// shared by host and device code.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eql_config.h"

namespace eqk {

// Lengths and first positions stay within 2^28 and packed rows below 2^29; a side
// of the window without a limit is 2^29, past every key from every position.
// Sums of three of them fit 32 bits.
constexpr int kAttnMaxPos = 1 << 28;
constexpr int kAttnNoLimit = 1 << 29;
constexpr int kAttnMaxD = 128;

// Workgroups of a grid over `pairs` head pairs of n items each (attn_item).
constexpr int kAttnFold = 16;
constexpr int64_t attn_blocks(int64_t pairs, int64_t n) {
  return n < kAttnFold ? pairs * n : pairs * 16 * (n / kAttnFold + 1);
}

// Waves that add a row's parts.
constexpr int attn_join_waves(int parts) { return parts > 8 ? 4 : 1; }

struct AttnArgs {
  const void *q, *k, *v, *go;
  void *o, *dq, *dk, *dv;
  const int *lengths, *starts;  // per sequence, or null
  float *lse, *delta;           // [B, Hkv, R], log2 units
  float* part;                  // fp32 parts of split rows or keys
  int64_t qs[3], ks[3], vs[3], os[3], gos[3], dqs[3], dks[3], dvs[3];  // elements: sequence, token, head
  int B, Lq, Lk, Hkv, G, R, D;
  int left, right, sinks;
  float scale, scale_log2e;
  int parts;                                        // forward: parts of a row's keys
  int key_tiles, sink_tiles, key_parts, sink_parts; // key/value gradient
  int run_tiles;                                    // row tiles that see a key tile
};

// streamed rows of a tile; a single wave stages by itself and holds half as many
constexpr int attn_tile(int dt) { return dt == kF32 ? 32 : 64; }
constexpr int attn_fwd_tile(int dt, int row_waves) { return row_waves == 1 ? 32 : attn_tile(dt); }
// Key waves of a workgroup of up to 32 rows: eight where they take all keys of their rows
// (8 sequences of 12 heads, 1,028 keys: 12 us, in parts and a join 19), four where
// the keys are split in parts (two workgroups a CU cover each other's joins).
constexpr int attn_key_waves(int parts) { return parts == 1 ? 8 : 4; }

// Row waves of a forward workgroup (4, or 1 beside several key waves), and the parts
// that the keys are split into.
struct AttnPlan {
  int waves, parts;
};
AttnPlan attn_plan(const AttnArgs& a, int dt, int cus);
size_t attn_part_bytes(const AttnArgs& a, const AttnPlan& p);
// Fills key_tiles .. sink_parts; returns the bytes of the parts.
constexpr int kAttnDkvKeys = 128;  // keys of a workgroup
size_t attn_dkv_plan(AttnArgs& a, int dt, int cus);

template <int DT>
hipError_t wattn_fwd(const AttnArgs& a, const AttnPlan& p, hipStream_t stream);
template <int DT>
hipError_t wattn_bwd(const AttnArgs& a, hipStream_t stream);
template <> hipError_t wattn_fwd<kF32>(const AttnArgs&, const AttnPlan&, hipStream_t);
template <> hipError_t wattn_fwd<kF16>(const AttnArgs&, const AttnPlan&, hipStream_t);
template <> hipError_t wattn_fwd<kBF16>(const AttnArgs&, const AttnPlan&, hipStream_t);
template <> hipError_t wattn_bwd<kF32>(const AttnArgs&, hipStream_t);
template <> hipError_t wattn_bwd<kF16>(const AttnArgs&, hipStream_t);
template <> hipError_t wattn_bwd<kBF16>(const AttnArgs&, hipStream_t);

}  // namespace eqk
