// C-ABI entry points of the decay attention: host-side validation and the layout of its workspace.
// See include/cotten_attn.h for the contract of every function.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/cotten_attn.h"
#include "cotten_decay_core.h"
#include "cotten_decay_launch.h"

namespace {

using cotten::decay::Args;
using cotten::decay::kChunk;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_shape(int B, int H, int N, int d_h, int dtype) {
  if (dtype != COTTEN_F32 && dtype != COTTEN_BF16 && dtype != COTTEN_F16) return COTTEN_ERR_BAD_DTYPE;
  if (B < 1 || H < 1 || N < 1) return COTTEN_ERR_BAD_SHAPE;
  if (d_h != 16 && d_h != 32 && d_h != 64 && d_h != 128) return COTTEN_ERR_UNSUPPORTED_HEAD_DIM;
  // (a slice takes four workgroups of up to 512 threads of a launch of less than 2^32)
  if (static_cast<long long>(B) * H > (1ll << 20) || N > (1 << 24)) return COTTEN_ERR_BAD_SHAPE;
  return COTTEN_OK;
}

// Floats of the workspace: local states of the segments, where sequences are cut, and partial sums of the decays' gradient.
struct Sizes {
  size_t states, counts, partial;
  cotten::decay::Segments segments;
  Sizes(int B, int H, int N, int d_h, int dtype, bool bwd, bool with_dg) {
    const size_t slices = static_cast<size_t>(B) * H;
    segments = cotten::decay::segments_of(static_cast<long long>(slices), (N + kChunk - 1) / kChunk, d_h, dtype, bwd);
    states = segments.count > 1 ? slices * segments.count * d_h * d_h : 0;
    counts = segments.count > 1 ? (2 * slices * segments.count + 3) / 4 * 4 : 0;
    partial = bwd && with_dg ? (2 * slices * segments.count * cotten::decay::waves_of(d_h) + 3) / 4 * 4 : 0;
  }
  size_t bytes(bool bwd, bool with_dg) const { return (states * (bwd ? with_dg ? 3 : 2 : 1) + counts + partial) * sizeof(float); }
};

// Checks what both directions share and fills the arguments.
int prepare(Args* a, const void* Q, const void* K, const void* V, const float* g, const uint8_t* mask, int B, int H, int N, int d_h,
            const cotten_decay_params* prm) {
  if (prm == nullptr || Q == nullptr || K == nullptr || V == nullptr || g == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (int rc = check_shape(B, H, N, d_h, prm->dtype)) return rc;
  const void* tensors[] = {Q, K, V, prm->workspace, prm->initial_state, prm->final_state, prm->dfinal_state, prm->dinitial_state};
  for (const void* t : tensors)
    if (!aligned16(t)) return COTTEN_ERR_MISALIGNED;
  if (reinterpret_cast<uintptr_t>(g) & 3u) return COTTEN_ERR_MISALIGNED;
  if (!std::isfinite(prm->scale) || !std::isfinite(prm->eps)) return COTTEN_ERR_BAD_PARAM;
  if (prm->layout != COTTEN_BHND && prm->layout != COTTEN_BNHD) return COTTEN_ERR_BAD_SHAPE;
  const long long e = prm->dtype == COTTEN_F32 ? 4 : 2, row = d_h * e;
  const bool heads_first = prm->layout == COTTEN_BHND;
  const long long stride_row = heads_first ? row : H * row;
  // the kernels address the rows of a slice, and those of a chunk beyond its end, with 31-bit byte offsets
  if ((N - 1ll) * stride_row + row >= (1ll << 31) || kChunk * stride_row >= (1ll << 31)) return COTTEN_ERR_BAD_SHAPE;
  a->stride_batch = static_cast<long long>(H) * N * row;
  a->stride_head = heads_first ? static_cast<long long>(N) * row : row;
  a->stride_row = static_cast<uint32_t>(stride_row);
  a->Q = static_cast<const unsigned char*>(Q);
  a->K = static_cast<const unsigned char*>(K);
  a->V = static_cast<const unsigned char*>(V);
  a->g = g;
  a->mask = mask;
  a->initial_state = prm->initial_state;
  a->H = H;
  a->N = N;
  a->chunks = (N + kChunk - 1) / kChunk;
  a->scale = prm->scale > 0.0f ? prm->scale : 1.0f;
  a->eps = prm->eps < 0.0f ? 1e-6f : prm->eps;
  return COTTEN_OK;
}

int use_workspace(Args* a, const Sizes& size, bool bwd, bool with_dg, const cotten_decay_params* prm) {
  a->segments = size.segments.count;
  a->segment_chunks = size.segments.chunks;
  const size_t need = size.bytes(bwd, with_dg);
  if (need == 0) return COTTEN_OK;
  if (prm->workspace == nullptr || prm->workspace_bytes < need) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  float* at = static_cast<float*>(prm->workspace);
  a->dg = reinterpret_cast<double*>(at);
  a->local_s = at + size.partial;
  a->local_d = a->local_s + size.states;
  a->local_t = bwd && with_dg ? a->local_d + size.states : nullptr;
  a->counts = a->local_s + size.states * (bwd ? with_dg ? 3 : 2 : 1);
  return COTTEN_OK;
}

}  // namespace

extern "C" {

size_t cotten_decay_workspace_bytes(int B, int H, int N, int d_h, int dtype, int is_bwd, int with_dg) {
  if (check_shape(B, H, N, d_h, dtype) != COTTEN_OK) return 0;
  return Sizes(B, H, N, d_h, dtype, is_bwd != 0, with_dg != 0).bytes(is_bwd != 0, with_dg != 0);
}

int cotten_decay_fwd(const void* Q, const void* K, const void* V, const float* g, const uint8_t* mask, void* O, int B, int H, int N,
                     int d_h, void* stream, const cotten_decay_params* params) {
  Args a{};
  if (O == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (int rc = prepare(&a, Q, K, V, g, mask, B, H, N, d_h, params)) return rc;
  if (!aligned16(O)) return COTTEN_ERR_MISALIGNED;
  a.O = static_cast<unsigned char*>(O);
  a.final_state = params->final_state;
  if (int rc = use_workspace(&a, Sizes(B, H, N, d_h, params->dtype, false, false), false, false, params)) return rc;
  return cotten::decay::launch_forward(a, params->dtype, d_h, B * H, static_cast<hipStream_t>(stream)) == hipSuccess ? COTTEN_OK
                                                                                                                   : COTTEN_ERR_LAUNCH;
}

int cotten_decay_bwd(const void* Q, const void* K, const void* V, const float* g, const uint8_t* mask, const void* dO, void* dQ,
                     void* dK, void* dV, float* dg, int B, int H, int N, int d_h, void* stream, const cotten_decay_params* params) {
  Args a{};
  if (dO == nullptr || dQ == nullptr || dK == nullptr || dV == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (int rc = prepare(&a, Q, K, V, g, mask, B, H, N, d_h, params)) return rc;
  if (!aligned16(dO) || !aligned16(dQ) || !aligned16(dK) || !aligned16(dV) || (reinterpret_cast<uintptr_t>(dg) & 3u)) return COTTEN_ERR_MISALIGNED;
  if (int rc = use_workspace(&a, Sizes(B, H, N, d_h, params->dtype, true, dg != nullptr), true, dg != nullptr, params)) return rc;
  a.dO = static_cast<const unsigned char*>(dO);
  a.dQ = static_cast<unsigned char*>(dQ);
  a.dK = static_cast<unsigned char*>(dK);
  a.dV = static_cast<unsigned char*>(dV);
  a.dfinal_state = params->dfinal_state;
  a.dinitial_state = params->dinitial_state;
  return cotten::decay::launch_backward(a, params->dtype, d_h, B * H, dg, static_cast<hipStream_t>(stream)) == hipSuccess ? COTTEN_OK
                                                                                                                       : COTTEN_ERR_LAUNCH;
}

}  // extern "C"
