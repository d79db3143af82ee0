// C-ABI entry points of the gated delta rule: host-side validation and the layout of its buffers.
// See include/cotten_attn.h for the contract of every function.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/cotten_attn.h"
#include "cotten_delta_core.h"
#include "cotten_delta_launch.h"

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_shape(int B, int H, int N, int d_h, int dtype) {
  if (dtype != COTTEN_F32 && dtype != COTTEN_BF16 && dtype != COTTEN_F16) return COTTEN_ERR_BAD_DTYPE;
  if (B < 1 || H < 1 || N < 1) return COTTEN_ERR_BAD_SHAPE;
  if (d_h != 16 && d_h != 32 && d_h != 64 && d_h != 128) return COTTEN_ERR_UNSUPPORTED_HEAD_DIM;
  // (a slice takes up to 768 threads of a launch of less than 2^32)
  if (static_cast<long long>(B) * H > (1ll << 22) || N > (1 << 24)) return COTTEN_ERR_BAD_SHAPE;
  return COTTEN_OK;
}

// Floats of the buffers: the state before (or the gradient after) every chunk, a row per token; and, where sequences are
// cut into segments, what each makes of a state (forward) and the gradient before each (backward).
struct Sizes {
  size_t states, rows, transitions, carries;
  cotten::delta::Segments segments;
  Sizes(int B, int H, int N, int d_h, int dtype) {
    const size_t slices = static_cast<size_t>(B) * H, state = static_cast<size_t>(d_h) * d_h;
    const size_t chunks = (static_cast<size_t>(N) + cotten::delta::kChunk - 1) / cotten::delta::kChunk;
    segments = cotten::delta::segments_of(static_cast<long long>(slices), static_cast<int>(chunks), d_h, dtype);
    states = slices * chunks * state;
    rows = slices * chunks * cotten::delta::kChunk * d_h;
    carries = segments.count > 1 ? slices * segments.count * state : 0;
    transitions = 2 * carries;
  }
  size_t kept() const { return (states + rows + transitions) * sizeof(float); }
  size_t backward(bool with_kept) const { return (states + rows + carries) * sizeof(float) + (with_kept ? 0 : kept()); }
  size_t forward(bool with_kept) const { return with_kept ? 0 : transitions * sizeof(float); }
};

// Checks what both directions share and fills the arguments.
int prepare(cotten::delta::Args* a, const void* Q, const void* K, const void* V, const float* g, const float* beta,
            const uint8_t* mask, int B, int H, int N, int d_h, const cotten_delta_params* prm) {
  if (prm == nullptr || Q == nullptr || K == nullptr || V == nullptr || g == nullptr || beta == nullptr)
    return COTTEN_ERR_NULL_POINTER;
  if (int rc = check_shape(B, H, N, d_h, prm->dtype)) return rc;
  const void* tensors[] = {Q, K, V, prm->workspace, prm->kept, prm->initial_state, prm->final_state, prm->dfinal_state,
                           prm->dinitial_state};
  for (const void* t : tensors)
    if (t != nullptr && !aligned16(t)) return COTTEN_ERR_MISALIGNED;
  if ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(beta)) & 3u) return COTTEN_ERR_MISALIGNED;
  if (!std::isfinite(prm->scale) || !std::isfinite(prm->eps)) return COTTEN_ERR_BAD_PARAM;
  if (prm->layout != COTTEN_BHND && prm->layout != COTTEN_BNHD) return COTTEN_ERR_BAD_SHAPE;
  // (one workgroup per chunk of 32 tokens, or two per slice)
  if (static_cast<long long>(B) * H * ((N + cotten::delta::kChunk - 1) / cotten::delta::kChunk) >= (1ll << 31))
    return COTTEN_ERR_BAD_SHAPE;
  const long long e = prm->dtype == COTTEN_F32 ? 4 : 2, row = d_h * e;
  const bool heads_first = prm->layout == COTTEN_BHND;
  const long long stride_row = heads_first ? row : H * row;
  // the kernels address the rows of a slice, and those of a chunk beyond its end, with 31-bit byte offsets
  if ((N - 1ll) * stride_row + row >= (1ll << 31) || cotten::delta::kChunk * stride_row >= (1ll << 31)) return COTTEN_ERR_BAD_SHAPE;
  a->stride_batch = static_cast<long long>(H) * N * row;
  a->stride_head = heads_first ? static_cast<long long>(N) * row : row;
  a->stride_row = static_cast<uint32_t>(stride_row);
  a->gate_batch = static_cast<long long>(H) * N;
  a->gate_head = heads_first ? N : 1;
  a->gate_row = heads_first ? 1 : H;
  a->Q = static_cast<const unsigned char*>(Q);
  a->K = static_cast<const unsigned char*>(K);
  a->V = static_cast<const unsigned char*>(V);
  a->g = g;
  a->beta = beta;
  a->mask = mask;
  a->initial_state = prm->initial_state;
  a->H = H;
  a->N = N;
  a->chunks = (N + cotten::delta::kChunk - 1) / cotten::delta::kChunk;
  a->scale = prm->scale > 0.0f ? prm->scale : 1.0f;
  a->eps = prm->eps < 0.0f ? 1e-6f : prm->eps;
  return COTTEN_OK;
}

void use_kept(cotten::delta::Args* a, float* at, const Sizes& size) {
  a->states = at;
  a->rows_u = at + size.states;
  a->transitions = a->rows_u + size.rows;
}

}  // namespace

extern "C" {

size_t cotten_delta_kept_bytes(int B, int H, int N, int d_h, int dtype) {
  return check_shape(B, H, N, d_h, dtype) == COTTEN_OK ? Sizes(B, H, N, d_h, dtype).kept() : 0;
}

size_t cotten_delta_workspace_bytes(int B, int H, int N, int d_h, int dtype, int is_bwd, int with_kept) {
  if (check_shape(B, H, N, d_h, dtype) != COTTEN_OK) return 0;
  const Sizes size(B, H, N, d_h, dtype);
  return is_bwd ? size.backward(with_kept != 0) : size.forward(with_kept != 0);
}

int cotten_delta_fwd(const void* Q, const void* K, const void* V, const float* g, const float* beta, const uint8_t* mask,
                     void* O, int B, int H, int N, int d_h, void* stream, const cotten_delta_params* params) {
  cotten::delta::Args a{};
  if (O == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (int rc = prepare(&a, Q, K, V, g, beta, mask, B, H, N, d_h, params)) return rc;
  if (!aligned16(O)) return COTTEN_ERR_MISALIGNED;
  a.O = static_cast<unsigned char*>(O);
  a.final_state = params->final_state;
  const Sizes size(B, H, N, d_h, params->dtype);
  a.segments = size.segments.count;
  a.segment_chunks = size.segments.chunks;
  if (params->kept != nullptr) {
    if (params->kept_bytes < size.kept()) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
    use_kept(&a, static_cast<float*>(params->kept), size);
  } else if (size.transitions != 0) {
    if (params->workspace == nullptr || params->workspace_bytes < size.forward(false)) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
    a.transitions = static_cast<float*>(params->workspace);
  }
  return cotten::delta::launch_forward(a, params->dtype, d_h, B * H, static_cast<hipStream_t>(stream)) == hipSuccess
             ? COTTEN_OK
             : COTTEN_ERR_LAUNCH;
}

int cotten_delta_bwd(const void* Q, const void* K, const void* V, const float* g, const float* beta, const uint8_t* mask,
                     const void* dO, void* dQ, void* dK, void* dV, float* dg, float* dbeta, int B, int H, int N, int d_h,
                     void* stream, const cotten_delta_params* params) {
  cotten::delta::Args a{};
  if (dO == nullptr || dQ == nullptr || dK == nullptr || dV == nullptr || dg == nullptr || dbeta == nullptr)
    return COTTEN_ERR_NULL_POINTER;
  if (int rc = prepare(&a, Q, K, V, g, beta, mask, B, H, N, d_h, params)) return rc;
  if (!aligned16(dO) || !aligned16(dQ) || !aligned16(dK) || !aligned16(dV)) return COTTEN_ERR_MISALIGNED;
  if ((reinterpret_cast<uintptr_t>(dg) | reinterpret_cast<uintptr_t>(dbeta)) & 3u) return COTTEN_ERR_MISALIGNED;
  const Sizes size(B, H, N, d_h, params->dtype);
  a.segments = size.segments.count;
  a.segment_chunks = size.segments.chunks;
  const bool kept = params->kept != nullptr;
  if (kept && params->kept_bytes < size.kept()) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  if (params->workspace == nullptr || params->workspace_bytes < size.backward(kept)) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  a.dstates = static_cast<float*>(params->workspace);
  a.rows_z = a.dstates + size.states;
  a.carries = a.rows_z + size.rows;
  use_kept(&a, kept ? static_cast<float*>(params->kept) : a.carries + size.carries, size);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (!kept && cotten::delta::launch_forward(a, params->dtype, d_h, B * H, s) != hipSuccess) return COTTEN_ERR_LAUNCH;
  a.dO = static_cast<const unsigned char*>(dO);
  a.dQ = static_cast<unsigned char*>(dQ);
  a.dK = static_cast<unsigned char*>(dK);
  a.dV = static_cast<unsigned char*>(dV);
  a.dg = dg;
  a.dbeta = dbeta;
  a.dfinal_state = params->dfinal_state;
  a.dinitial_state = params->dinitial_state;
  return cotten::delta::launch_backward(a, params->dtype, d_h, B * H, s) == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

}  // extern "C"
