// Launchers of the gated delta rule's kernels: arguments are validated (cotten_delta_api.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace cotten {
namespace delta {

struct Args;

// O, final_state, states and rows_u, each where its pointer is given.
hipError_t launch_forward(const Args& a, int dtype, int D, int slices, hipStream_t stream);
// dQ, dK, dV, dg, dbeta and dinitial_state from states and rows_u; uses dstates and rows_z.
hipError_t launch_backward(const Args& a, int dtype, int D, int slices, hipStream_t stream);

}  // namespace delta
}  // namespace cotten
