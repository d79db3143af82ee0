// Launchers of the decay attention's kernels: arguments are validated (cotten_decay_api.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace cotten {
namespace decay {

struct Args;

// Into how many segments of how many chunks the sequences of a call are cut: a workgroup walks its chunks one after the
// other, so few slices of long sequences leave the device idle.  A first launch walks the segments for what each adds to the
// state, and the rows then follow from the sum over the segments before.
struct Segments {
  int count, chunks;
};
Segments segments_of(long long slices, int chunks, int D, int dtype, bool bwd);

hipError_t launch_forward(const Args& a, int dtype, int D, int slices, hipStream_t stream);
// dg: [H], or nullptr where the decays are not trained; partial sums go through a.dg.
hipError_t launch_backward(const Args& a, int dtype, int D, int slices, float* dg, hipStream_t stream);
inline int waves_of(int D) { return D / 16; }

}  // namespace decay
}  // namespace cotten
