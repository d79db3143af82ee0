// Launchers of the gated delta rule's kernels: arguments are validated (cotten_delta_api.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace cotten {
namespace delta {

struct Args;

// Into how many segments of how many chunks the sequences of a call are cut.
//
// A workgroup walks its chunks one after the other, so few slices of long sequences leave the device idle.  A segment is
// linear in the state before it, S' = M S + R: a first launch walks the segments for R (from a zero state) and M (from unit
// columns, without V), and the segments' outputs then follow from the states before them, each M S + R once per
// segment before.  That is twice to three times the work, in chunks / segments steps instead of chunks.
struct Segments {
  int count, chunks;
};
Segments segments_of(long long slices, int chunks, int D, int dtype);

// O, final_state, states and rows_u, each where its pointer is given.
hipError_t launch_forward(const Args& a, int dtype, int D, int slices, hipStream_t stream);
// dQ, dK, dV, dg, dbeta and dinitial_state from states and rows_u; uses dstates and rows_z.
hipError_t launch_backward(const Args& a, int dtype, int D, int slices, hipStream_t stream);

}  // namespace delta
}  // namespace cotten
