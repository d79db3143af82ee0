// Kernels of the decay attention (cotten_decay_core.h has the formulas): a recurrence for a few tokens, and chunks of 32 tokens
// on the matrix cores for more.
#include "cotten_decay_core.h"
#include "cotten_decay_launch.h"
#include "cotten_launch.h"

namespace cotten {
namespace decay {
namespace {

extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

// ---- token by token -----------------------------------------------------------------------------------------------
//
// A wave carries up to 32 columns of a state in registers, eight lanes to a row of 128 bytes, the rows dealt to the lane groups;
// q^ . S is a sum over the groups by lane permutes.  One token is bound by the state, read and written once: 4096 x 2 states of 64 x 64
// in 40.6 us, 6.6 TB/s (the memory-side cache helps); 512 x 4 in 9.6.
template <class E, int D>
__global__ __launch_bounds__(256) void step_kernel(Args a, int parts) {
  constexpr int kCols = D < 32 ? D : 32;         // columns of a wave
  constexpr int kLanes = kCols / 4;              // lanes of a row
  constexpr int kGroups = 64 / kLanes;
  constexpr int kRows = D / kGroups;             // rows of a lane: group, group + kGroups, ...
  static_assert(D % kGroups == 0, "rows are dealt evenly");
  const int lane = threadIdx.x & 63;
  const long long unit = static_cast<long long>(blockIdx.x) * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= static_cast<long long>(parts) * (D / kCols)) return;
  const int slice = static_cast<int>(unit / (D / kCols)), col = static_cast<int>(unit % (D / kCols)) * kCols + 4 * (lane % kLanes);
  const int group = lane / kLanes;
  const Slice s(a, slice, D * E::kBytes);
  const __amdgpu_buffer_rsrc_t Q = s.of(a.Q, 0, a.stride_row), K = s.of(a.K, 0, a.stride_row), V = s.of(a.V, 0, a.stride_row),
                               O = s.of(a.O, 0, a.stride_row);
  f32x4_t S[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    S[r] = a.initial_state == nullptr
               ? f32x4_t{0, 0, 0, 0}
               : *reinterpret_cast<const f32x4_t*>(a.initial_state + (static_cast<long long>(slice) * D + group + r * kGroups) * D + col);
  // Near 1 (weak) the decay of a call's tokens is left for its end, a^p in two floats, and what a token adds is divided by a^p before: a server makes
  // one call after the other, and the rounding of a factor would be the same in every one of them.  Other decays leave nothing for roundings to add up in.
  const double rate = rate_of(s.g), whole = exp2(rate);
  const bool weak = whole > 0.5 && whole < 2.0;
  const float now = weak ? 1.0f : static_cast<float>(whole);
  int count = 0;
  for (int t = 0; t < a.N; ++t) {
    const bool live = s.mask == nullptr || s.mask[t] != 0;
    const uint32_t row = static_cast<uint32_t>(t) * a.stride_row;
    const f32x4_t v = E::load_four(V, live ? row + col * E::kBytes : kNowhere);
    float k[kRows], q[kRows], kk = 0.0f, qq = 0.0f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const uint32_t off = row + (group + r * kGroups) * E::kBytes;
      k[r] = E::value(E::load_one(K, live ? off : kNowhere));
      q[r] = E::value(E::load_one(Q, off));
      kk = fmaf(k[r], k[r], kk);
      qq = fmaf(q[r], q[r], qq);
    }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
      kk += __shfl_xor(kk, m);
      qq += __shfl_xor(qq, m);
    }
    count += live ? 1 : 0;
    const float later = weak ? static_cast<float>(rate * static_cast<double>(count)) : 0.0f;
    const float rk = live ? __builtin_amdgcn_rsqf(kk + a.eps) * __builtin_amdgcn_exp2f(-later) : 0.0f;
    const float rq = a.scale * __builtin_amdgcn_rsqf(qq + a.eps) * __builtin_amdgcn_exp2f(later), decay = live ? now : 1.0f;
    f32x4_t o = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const float unit_k = k[r] * rk;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        S[r][c] = fmaf(unit_k, v[c], S[r][c] * decay);
        o[c] = fmaf(q[r], S[r][c], o[c]);
      }
    }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += __shfl_xor(o[c], m);
    if (group == 0) E::store_four(O, row + col * E::kBytes, o * rq);
  }
  if (a.final_state != nullptr) {
    if (weak && count != 0) {
      const double left = exp2(rate * static_cast<double>(count));
      const float hi = static_cast<float>(left), lo = static_cast<float>(left - static_cast<double>(hi));
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) S[r][c] = fmaf(S[r][c], hi, S[r][c] * lo);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      *reinterpret_cast<f32x4_t*>(a.final_state + (static_cast<long long>(slice) * D + group + r * kGroups) * D + col) = S[r];
  }
}

// ---- chunks ---------------------------------------------------------------------------------------------------------
//
// One walk, made for what it writes (see walk() in cotten_decay_core.h): the columns of a state are dealt to waves of 16, so a state and the
// products with it need no exchange, and a chunk costs two barriers: one behind its rows, one behind the products of its pairs, which the
// waves share.  128 x 4 slices of 200 x 64 bf16: forward 16 us (52 MB, 3.3 TB/s), backward without dg 39 (92 MB; three walks, each with
// its own reads, most of them found in L2).  From 768 slices on a forward moves 4.6 to 5.1 TB/s, a backward 2.6: three workgroups a compute unit keep
// the vector units busy with cutting rows and states into pieces; with one, a chunk takes 1.35 us, its own chain of LDS, products and
// barriers.  Rows in two places of LDS with one barrier a chunk, and two chunks of rows ahead, were built: 16.2 to 17.8 us, 15.4 to 16.7.

// Waves on a SIMD that the registers of a walk leave room for.
template <class E, int D, bool DECAYS = false>
constexpr int kRoom = E::kBytes == 2 && D <= 64 && !DECAYS ? 3 : 2;

template <class E, int D, int ROLE>
__global__ __launch_bounds__(64 * kWaves<D>, (kRoom<E, D, ROLE == kDecays>)) void walk_kernel(Args a) {
  walk<E, D, ROLE>(a, blockIdx.x, smem);
}

// d = 128: two workgroups of four waves a unit, half of the columns each, eight apart for the same reason as the roles below.  Each loads all
// rows, but a wave has the registers of a SIMD to itself (eight waves, two a SIMD, spill 89 of fp32's), and nobody waits for eight.
template <class E, int D, int ROLE>
__global__ __launch_bounds__(64 * kWaves<D> / 2) void halves_kernel(Args a, int units) {
  const int turn = blockIdx.x / 16, rest = blockIdx.x % 16, unit = turn * 8 + rest % 8;
  if (unit < units) walk<E, D, ROLE, 2>(a, unit, smem, rest / 8);
}

// The backward's walks as roles of one launch.  Workgroups go to the eight XCDs in turn: the roles of a unit are eight apart,
// so they find each other's rows in one L2.
template <class E, int D>
__global__ __launch_bounds__(64 * kWaves<D>, (kRoom<E, D>)) void grad_kernel(Args a, int units) {
  const int turn = blockIdx.x / 24, rest = blockIdx.x % 24, role = rest / 8, unit = turn * 8 + rest % 8;
  if (unit >= units) return;
  if (role == 0) walk<E, D, kDq>(a, unit, smem);
  else if (role == 1) walk<E, D, kDk>(a, unit, smem);
  else walk<E, D, kDv>(a, unit, smem);
}
// ... with keys and values in one.
template <class E, int D>
__global__ __launch_bounds__(64 * kWaves<D>, (kRoom<E, D>)) void joined_grad_kernel(Args a, int units) {
  const int turn = blockIdx.x / 16, rest = blockIdx.x % 16, unit = turn * 8 + rest % 8;
  if (unit >= units) return;
  if (rest / 8 == 0) walk<E, D, kDq>(a, unit, smem);
  else walk_back<E, D>(a, unit, smem);
}

// What the segments add to S (with its derivative by g) and to dS.
template <class E, int D, bool DERIVATIVES>
__global__ __launch_bounds__(64 * kWaves<D>, 2) void grad_states_kernel(Args a, int units) {
  if (static_cast<int>(blockIdx.x) < units) walk<E, D, DERIVATIVES ? kStatesAndDerivatives : kStates>(a, blockIdx.x, smem);
  else walk<E, D, kGradStates>(a, blockIdx.x - units, smem);
}

// From what every segment adds to the states before (behind) all: four values of a slice's states a thread, from segment to segment.
// `back`: the gradients, from the last to the first, by workgroups behind the first `forwards`.
constexpr int kScanThreads = 256, kScanAhead = 8;
__global__ __launch_bounds__(kScanThreads) void scan_kernel(Args a, int state_quads, long long quads, unsigned forwards) {
  const bool back = blockIdx.x >= forwards;
  const long long i = static_cast<long long>(blockIdx.x - (back ? forwards : 0u)) * kScanThreads + threadIdx.x;
  if (i >= quads) return;
  const long long slice = i / state_quads, at = slice * a.segments * state_quads + (i - slice * state_quads);
  const float* counts = a.counts + 2 * slice * a.segments;
  f32x4_t* s = reinterpret_cast<f32x4_t*>(back ? a.local_d : a.local_s) + at;
  f32x4_t* t = a.local_t == nullptr || back ? nullptr : reinterpret_cast<f32x4_t*>(a.local_t) + at;
  const int last = a.segments - 1;
  f32x4_t state = s[static_cast<long long>(last) * state_quads], derivative = {0, 0, 0, 0};
  for (int base = 0; base < last; base += kScanAhead) {
    f32x4_t ds[kScanAhead], dt[kScanAhead];
    float n[kScanAhead], w[kScanAhead];
#pragma unroll
    for (int u = 0; u < kScanAhead; ++u) {
      const int j = base + u < last ? base + u : last - 1, segment = back ? last - 1 - j : j;
      ds[u] = s[static_cast<long long>(segment) * state_quads];
      if (t != nullptr) dt[u] = t[static_cast<long long>(segment) * state_quads];
      n[u] = counts[2 * segment];
      w[u] = counts[2 * segment + 1];
    }
#pragma unroll
    for (int u = 0; u < kScanAhead; ++u) {
      const int j = base + u, segment = back ? last - 1 - j : j;
      if (j >= last) break;
      s[static_cast<long long>(segment) * state_quads] = state;
      if (back) {
        state = state * w[u] + ds[u];   // (the first segment's is nothing, and goes nowhere)
      } else {
        if (t != nullptr) {
          t[static_cast<long long>(segment) * state_quads] = derivative;
          derivative = j == 0 ? dt[u] : w[u] * (derivative + n[u] * state) + dt[u];
        }
        state = j == 0 ? ds[u] : state * w[u] + ds[u];   // (the first segment's has the initial state in it)
      }
    }
  }
  if (!back) {
    s[static_cast<long long>(last) * state_quads] = state;
    if (t != nullptr) t[static_cast<long long>(last) * state_quads] = derivative;
  }
}
void launch_scan(const Args& a, int slices, int D, bool both, hipStream_t stream) {
  const int quads = D * D / 4;
  const long long all = static_cast<long long>(slices) * quads;
  const unsigned blocks = static_cast<unsigned>((all + kScanThreads - 1) / kScanThreads);
  scan_kernel<<<dim3(both ? 2 * blocks : blocks), dim3(kScanThreads), 0, stream>>>(a, quads, all, blocks);
}

// dg of a head (4 us for 128 sequences' sums of eight parts): every thread sums some of its slices' partial sums, in the order that it finds them, and the threads are joined.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void sum_decays_kernel(const double* partial, float* dg, int B, int H, int of_slice) {
  __shared__ double of_wave[kSumThreads / 64];
  const int h = blockIdx.x;
  const long long n = static_cast<long long>(B) * of_slice;
  double s = 0.0;
#pragma unroll 4
  for (long long i = threadIdx.x; i < n; i += kSumThreads) {
    const long long b = i / of_slice;
    s += partial[(b * H + h) * of_slice + (i - b * of_slice)];
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSumThreads / 64; ++w) s += of_wave[w];
    dg[h] = static_cast<float>(s);
  }
}

constexpr int greatest(int a, int b) { return a > b ? a : b; }

template <class Kernel>
hipError_t granted(Kernel kernel, int bytes) {
  return bytes > 64 * 1024 ? grant_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes) : hipSuccess;
}

// Up to how many tokens the recurrence is as fast as a chunk of 32, which takes the same for any number of them.  us, recurrence / chunk:
//   bf16 d = 64, 2048 slices  5 tokens 14.6 / 15.2, 6 16.8 / 15.5     fp16 d = 128, 512 slices  6 tokens 17.8 / 17.8, 8 21.5 / 17.4; 2048  8 57 / 67
//   bf16 d = 16, 8192         5 tokens 14.6 / 15.5, 6 16.7 / 15.6     fp32 d = 128, 512  8 tokens 20.3 / 21.4, 12 26.1 / 21.7; 2048  12 66 / 76
//   fp32 d = 32, 2048        12 tokens 11.3 / 12.4, 16 13.8 / 12.6; 8192  12 29.8 / 34.2, 16 36.2 / 34.1
template <class E, int D>
constexpr int kMostSteps = E::kBytes == 4 ? (D == 128 ? 10 : 12) : (D == 128 ? 6 : 5);

// The decays' walk.  At d = 128 as halves where both find a compute unit of their own: the backward of 128 slices of 197 tokens takes 97 us
// that way and 106 with eight waves in fp16, 75 and 77 in bf16; of 256 slices, two rounds, 160 and 139, 122 and 100.  fp32's are halves at any
// number: 128 slices 121 and 152, 256 slices 200 and 212, 1024 slices 798 and 849, 64 slices of 2048 tokens 685 and 946 (at 192 slices no faster).
// (The forward walk was tried as well: 1 us faster up to 128 slices, 4 to 20 % slower in segments.)
template <class E, int D>
hipError_t launch_decays(const Args& a, int units, hipStream_t s) {
  constexpr int kBytes = kLds<E, D, kDecays>, kMostHalved = D != 128 ? 0 : E::kBytes == 4 ? 0x7fffffff : 128;
  if constexpr (kMostHalved > 0) {
    if (units <= kMostHalved) {
      if (hipError_t rc = granted(halves_kernel<E, D, kDecays>, kBytes)) return rc;
      halves_kernel<E, D, kDecays><<<dim3(static_cast<unsigned>((units + 7) / 8) * 16u), dim3(32 * kWaves<D>), kBytes, s>>>(a, units);
      return hipSuccess;
    }
  }
  if constexpr (kMostHalved < 0x7fffffff) {
    if (hipError_t rc = granted(walk_kernel<E, D, kDecays>, kBytes)) return rc;
    walk_kernel<E, D, kDecays><<<dim3(static_cast<unsigned>(units)), dim3(64 * kWaves<D>), kBytes, s>>>(a);
  }
  return hipSuccess;
}

// The walks of dQ, dK and dV.  At d = 128 a compute unit has room for one workgroup, and 16-bit walks take as many rounds as the workgroups need:
// three of a unit, or two of which the joint one takes half as long again.  us, three / two: fp16 64 x 197 tokens 30.9 / 45.0, 128 x 197 58.4 / 47.9, 200 x 197
// 84.5 / 88, 512 x 197 171 / 174, 16 x 2048 in 8 segments 97.8 / 82.7; bf16 25 / 35, 46.5 / 36.6, 64 / 67, 129 / 130, 75 / 63.  (Narrower rows,
// several workgroups to a compute unit, are no faster joined: bf16 d = 64, 512 x 200 45 / 48, 4096 x 200 307 / 299, fp16 413 / 462.)
template <class E, int D>
hipError_t launch_gradients(const Args& a, int units, hipStream_t s) {
  const unsigned eights = static_cast<unsigned>((units + 7) / 8);
  constexpr int kUnits = 256;  // compute units
  const auto rounds = [](long long workgroups) { return (workgroups + kUnits - 1) / kUnits; };
  if constexpr (D == 128 && E::kBytes == 2) {
    if (3 * rounds(2ll * units) < 2 * rounds(3ll * units)) {
      constexpr int kBytes = greatest(kLds<E, D, kDq>, BackPlace<E, D>::kBytes);
      static_assert(kBytes <= 160 * 1024, "a workgroup's LDS");
      if (hipError_t rc = granted(joined_grad_kernel<E, D>, kBytes)) return rc;
      joined_grad_kernel<E, D><<<dim3(eights * 16u), dim3(64 * kWaves<D>), kBytes, s>>>(a, units);
      return hipSuccess;
    }
  }
  constexpr int kBytes = greatest(kLds<E, D, kDq>, kLds<E, D, kDv>);
  if (hipError_t rc = granted(grad_kernel<E, D>, kBytes)) return rc;
  grad_kernel<E, D><<<dim3(eights * 24u), dim3(64 * kWaves<D>), kBytes, s>>>(a, units);
  return hipSuccess;
}

// A forward's segments sum the states before them themselves, in place of a launch that does it for all, where there is little to read for as many
// workgroups as there are: up to five, states of d = 16, and of d = 32 unless all compute units are busy with it (few slices leave a scan few
// workgroups, which walk the segments one after the other).  us, scan / sums:
//   d = 64 bf16   4 x 400 (5 segments) 16.2 / 13.4, 128 x 1024 (4) 35.7 / 31.8, 64 x 1024 (8) 24.3 / 27.4     128 fp16  64 x 1024 (4) 66.8 / 59, 4 x 1024 (16) 26 / 35
//   d = 32 bf16   4 x 4096 (32) 19.9 / 16.5, 32 x 2048 (32) 21.3 / 22.8, 8 x 16384 (64) 35.4 / 32.3, 16 x 16384 (64) 38.8 / 42.5, 8 x 32768 (128) 48.7 / 55.3,
//                 1 x 65536 (256) 60.6 / 50.9, 4 x 65536 (256) 68.6 / 79.7, 1 x 2^20 (1026) 230 / 195; fp32  64 x 1024 (16) 24.4 / 24.6, 4 x 65536 84.7 / 93.7
//   d = 16 bf16   32 x 4096 (32) 22.6 / 18.8, 16 x 16384 (64) 35.1 / 29.4, 4 x 65536 (258) 62.5 / 48.9, 1 x 2^20 (2064, as many as there are) 321 / 247
bool sums_of_its_own(int D, long long slices, int segments) {
  return segments <= 5 || D == 16 || (D == 32 && (slices < 4 || slices * segments <= 512));
}
template <class E, int D>
hipError_t forward(Args a, int slices, hipStream_t s) {
  if (a.N <= kMostSteps<E, D>) {
    constexpr int kParts = D < 32 ? 1 : D / 32;
    const long long waves = static_cast<long long>(slices) * kParts;
    const int of_block = waves > 4096 ? 4 : 1;
    step_kernel<E, D><<<dim3(static_cast<unsigned>((waves + of_block - 1) / of_block)), dim3(64 * of_block), 0, s>>>(a, slices);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>(slices) * a.segments), block(64 * kWaves<D>);
  if (a.segments > 1) {
    constexpr int kBytes = kLds<E, D, kStates>;
    if (hipError_t rc = granted(walk_kernel<E, D, kStates>, kBytes)) return rc;
    walk_kernel<E, D, kStates><<<grid, block, kBytes, s>>>(a);
    a.unscanned = sums_of_its_own(D, slices, a.segments);
    if (!a.unscanned) launch_scan(a, slices, D, false, s);
  }
  constexpr int kBytes = kLds<E, D, kOut>;
  if (hipError_t rc = granted(walk_kernel<E, D, kOut>, kBytes)) return rc;
  walk_kernel<E, D, kOut><<<grid, block, kBytes, s>>>(a);
  return hipGetLastError();
}

template <class E, int D>
hipError_t backward(const Args& a, int slices, float* dg, hipStream_t s) {
  const int units = slices * a.segments;
  const dim3 block(64 * kWaves<D>);
  if (a.segments > 1) {
    constexpr int kBytes = kLds<E, D, kStates>;
    const auto kernel = dg != nullptr ? grad_states_kernel<E, D, true> : grad_states_kernel<E, D, false>;
    if (hipError_t rc = granted(kernel, kBytes)) return rc;
    kernel<<<dim3(2u * units), block, kBytes, s>>>(a, units);
    launch_scan(a, slices, D, true, s);
  }
  if (hipError_t rc = launch_gradients<E, D>(a, units, s)) return rc;
  if (dg != nullptr) {
    // (a launch of its own: it needs the most registers, and would take them from the other roles)
    if (hipError_t rc = launch_decays<E, D>(a, units, s)) return rc;
    sum_decays_kernel<<<dim3(a.H), dim3(kSumThreads), 0, s>>>(a.dg, dg, slices / a.H, a.H, a.segments * kWaves<D>);
  }
  return hipGetLastError();
}

template <class E>
hipError_t forward(const Args& a, int D, int slices, hipStream_t s) {
  return D == 16 ? forward<E, 16>(a, slices, s) : D == 32 ? forward<E, 32>(a, slices, s) : D == 64 ? forward<E, 64>(a, slices, s) : forward<E, 128>(a, slices, s);
}
template <class E>
hipError_t backward(const Args& a, int D, int slices, float* dg, hipStream_t s) {
  return D == 16   ? backward<E, 16>(a, slices, dg, s)
         : D == 32 ? backward<E, 32>(a, slices, dg, s)
         : D == 64 ? backward<E, 64>(a, slices, dg, s)
                   : backward<E, 128>(a, slices, dg, s);
}

}  // namespace

// Segments for 2048 waves of a forward and 1024 of a backward (whose rows take three walks), of two chunks at least, where that makes
// three or more: the states' own walk is half of the rows', so two gain nothing.  us, whole / three / four / eight / sixteen / 32 segments:
//   bf16 d = 64, 4 x 4096 rows     forward 173 / 99 / 77 / 44 / 29 / 24      backward 216 / 112 / 87 / 50 / 33 / 29
//                64 x 4096                 170 / 101 / 80 / 56 / 53 / 65             216 / 162 / 128 / 121 / 128 / 149
//               128 x 1024                  46 / 42 / 37 / 37 / 49                    68 / 77 / 73 / 81 / 99
//               256 x 1024                  46 / 54 / 56 / 65                         88 / 127 / 131 / 151
//   fp32 d = 32, 128 x 1024                 63 / 48 / 39 / 31 / 36                    83 / 64 / 66 / 62 / 67
//   fp16 d = 128, 64 x 1024                109 / 80 / 67 / 78 / 99                   125 / 195 / 160 / 181 / 228
// Sequences of few chunks gain nothing: bf16 d = 64, 4 x 256 rows 14.1 / 16.1 / 15.2, fp32 20.9 / 20.2 / 17.1, fp16 d = 128 31.1 / 26.9 / 21.5;
// bf16 4 x 512 24.4 / 22.2 / 18.4 / 15.1.  (All forwards with a scan; where they do without, they take 2 to 4 us less.)
Segments segments_of(long long slices, int chunks, int D, int dtype, bool bwd) {
  const int least = dtype != 0 && D <= 64 ? 10 : 7, cap = chunks / 8 > 32 ? chunks / 8 : 32;
  long long count = (bwd ? 1024 : 2048) / (slices * waves_of(D));
  if (count > chunks / 2) count = chunks / 2;
  if (count > cap) count = cap;
  if (chunks < least || count < 3) return {1, chunks};
  const int each = static_cast<int>((chunks + count - 1) / count);
  return {(chunks + each - 1) / each, each};
}

hipError_t launch_forward(const Args& a, int dtype, int D, int slices, hipStream_t stream) {
  return dtype == 0 ? forward<delta::F32>(a, D, slices, stream) : dtype == 1 ? forward<delta::Bf16>(a, D, slices, stream) : forward<delta::F16>(a, D, slices, stream);
}
hipError_t launch_backward(const Args& a, int dtype, int D, int slices, float* dg, hipStream_t stream) {
  return dtype == 0   ? backward<delta::F32>(a, D, slices, dg, stream)
         : dtype == 1 ? backward<delta::Bf16>(a, D, slices, dg, stream)
                      : backward<delta::F16>(a, D, slices, dg, stream);
}

}  // namespace decay
}  // namespace cotten
