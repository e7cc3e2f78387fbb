// eql_encoder.h -- launches of the rotary and group-norm kernels.  Host code only.
#pragma once
#include "eql_gnact.h"
#include "eql_rotary.h"

namespace eqk {

hipError_t launch_rotary(int dt, const RotaryArgs& a, int vec, hipStream_t stream);
// Fills hold and threads, chunks, cblocks, rows and width for vectors of `vec` elements.
void gn_plan(GnArgs& a, int vec, int cus, bool bwd);
hipError_t launch_gn_forward(int dt, const GnArgs& a, int vec, hipStream_t stream);
hipError_t launch_gn_backward(int dt, const GnArgs& a, int vec, hipStream_t stream);

}  // namespace eqk
