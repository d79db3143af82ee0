// The seam between two blocks and dropout by itself:
//
//     Y = X + alpha * gate * drop(N(F; w1, b1))          H = N(Y; w2, b2)
//     N(x; w, b) = (x - mu) r w + b,   r = 1 / sqrt(mean (x - mu)^2 + eps),   mu = mean x (layer) or 0 (rms)
//
// and, with d = dY + (the gradient of Y through H), y^ and f^ the normalised rows and z what is added:
//
//     d = dY + r2 (a - y^ mean(a y^) - mean(a) [layer]),  a = dH w2       dw2 = sum dH y^     db2 = sum dH
//     dX = d      dgate = sum alpha d z      e = drop(alpha d gate)       dw1 = sum e f^      db1 = sum e
//     dF = r1 (e w1 - f^ mean(e w1 f^) - mean(e w1) [layer])
//
// Everything here moves memory: a row is read once and stays in the registers of the lanes that share it, the backward makes
// the forward's rows again from X and F (nothing is kept, and H's row is not rounded on the way), and the mask of the
// dropout is drawn again where it is needed.  Sums over a row and over rows are fp32, each result is rounded once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/cotten_attn.h"
#include "cotten_philox.h"

namespace cotten {
namespace residual {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ---- eight elements of a row ---------------------------------------------------------------------------------------

// ALIGNED: pieces begin at 16-byte boundaries.  WHOLE: none is short (rows of a multiple of eight elements).
template <int ALIGN>
struct Word;
template <>
struct Word<2> { typedef u32x4_t __attribute__((aligned(2))) type; };
template <>
struct Word<4> { typedef u32x4_t __attribute__((aligned(4))) type; };
template <>
struct Word<16> { typedef u32x4_t type; };

template <class T>
struct Raw {
  u32x4_t w[sizeof(T) / 2];
};
template <class T, bool ALIGNED, bool WHOLE = ALIGNED>
__device__ __forceinline__ Raw<T> load(const T* p, int valid) {
  typedef typename Word<ALIGNED ? 16 : sizeof(T)>::type word;
  Raw<T> r;
  if (WHOLE ? valid > 0 : valid >= 8) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const word*>(p)[i];
  } else {
    T x[8] = {};
    if constexpr (!WHOLE)
      for (int i = 0; i < 7; ++i)
        if (i < valid) x[i] = p[i];
    __builtin_memcpy(&r, x, sizeof(r));
  }
  return r;
}
template <class T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&x)[8]) {
  T e[8];
  __builtin_memcpy(e, &r, sizeof(r));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(e[i]);
}
template <class T, bool ALIGNED, bool WHOLE = ALIGNED>
__device__ __forceinline__ void store(T* p, const float (&x)[8], int valid) {
  typedef typename Word<ALIGNED ? 16 : sizeof(T)>::type word;
  T e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = static_cast<T>(x[i]);
  if (WHOLE ? valid > 0 : valid >= 8) {
    Raw<T> r;
    __builtin_memcpy(&r, e, sizeof(r));
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<word*>(p)[i] = r.w[i];
  } else if constexpr (!WHOLE) {
    for (int i = 0; i < 7; ++i)
      if (i < valid) p[i] = e[i];
  }
}

// ---- dropout --------------------------------------------------------------------------------------------------------

constexpr int kThreads = 256;
constexpr int kDropPieces = 2;  // of a thread, on their way together

// y = x * factor where it is kept, 0 elsewhere (whatever x holds there).  The same call on the upstream gradient is the backward.
// Bound by memory, read and written once: 1024 x 200 x 256 bf16 (210 MB) in 38 us, 5.4 TB/s with what the memory-side cache holds; ten rounds of
// the generator for eight elements hide behind it.  Two pieces a thread, or a wave waits for one load at a time.
template <class T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, T* y, uint64_t n, Drop drop) {
  const Lots lots(drop);
  const uint64_t pieces = (n + 7) >> 3;
  for (uint64_t first = static_cast<uint64_t>(blockIdx.x) * (kThreads * kDropPieces) + threadIdx.x; first < pieces;
       first += static_cast<uint64_t>(gridDim.x) * (kThreads * kDropPieces)) {
    Raw<T> raw[kDropPieces];
    int valid[kDropPieces];
#pragma unroll
    for (int u = 0; u < kDropPieces; ++u) {
      const uint64_t piece = first + u * kThreads;
      valid[u] = piece >= pieces ? 0 : n - piece * 8 < 8 ? static_cast<int>(n - piece * 8) : 8;
      raw[u] = load<T, true, false>(x + piece * 8, valid[u]);
    }
#pragma unroll
    for (int u = 0; u < kDropPieces; ++u) {
      const uint64_t piece = first + u * kThreads;
      const u32x4_t w = lots.draw(piece);
      float v[8];
      unpack<T>(raw[u], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = lots.keeps(w, i) ? v[i] * lots.factor : 0.0f;
      store<T, true, false>(y + piece * 8, v, valid[u]);
    }
  }
}

// ---- rows -----------------------------------------------------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), CTRL, 0xF, 0xF, true));
}
// Sum over the LANES lanes of a group, in all of them.
template <int LANES>
__device__ __forceinline__ float sum_of_lanes(float x) {
  x = add_dpp<0xB1>(x);                          // quad_perm 1,0,3,2
  x = add_dpp<0x4E>(x);                          // quad_perm 2,3,0,1
  x = add_dpp<0x141>(x);                         // row_half_mirror: the other four of eight
  if constexpr (LANES > 8) x = add_dpp<0x140>(x);  // row_mirror: the other eight of sixteen
  if constexpr (LANES > 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if constexpr (LANES > 32) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  }
  return x;
}

// The lanes that share a row: a part of a wave, or all waves of a workgroup.  A piece of eight elements a lane: two held twice the
// registers, and a second wave on a SIMD hides more of the memory's latency than a second piece.
template <int LANES_>
struct Shape {
  static constexpr int kLanes = LANES_, kPieces = 1;
  static constexpr int kBlock = LANES_ > 64 ? LANES_ : kThreads;
  static constexpr int kWaves = LANES_ / 64;         // of a row
  static constexpr int kGroups = kBlock / LANES_;    // rows that a workgroup has under way
  static constexpr int kMost = LANES_ * kPieces * 8; // elements of a row
};

// Sums over a row, two at a time.  Across waves through LDS, in two buffers by turns: a wave writes one again when all
// have passed the barrier behind their reads of it.
template <class S>
struct RowSums {
  float* at;
  int turn = 0;
  __device__ __forceinline__ void operator()(float& x, float& y) {
    x = sum_of_lanes<S::kLanes < 64 ? S::kLanes : 64>(x);
    y = sum_of_lanes<S::kLanes < 64 ? S::kLanes : 64>(y);
    if constexpr (S::kWaves > 1) {
      float* to = at + turn * 2 * S::kWaves;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
        to[2 * (threadIdx.x >> 6)] = x;
        to[2 * (threadIdx.x >> 6) + 1] = y;
      }
      __syncthreads();
      x = y = 0.0f;
#pragma unroll
      for (int w = 0; w < S::kWaves; ++w) {
        x += to[2 * w];
        y += to[2 * w + 1];
      }
    }
  }
  __device__ __forceinline__ void operator()(float& x) {
    if constexpr (S::kWaves > 1) {
      float y = 0.0f;
      (*this)(x, y);
    } else {
      x = sum_of_lanes<S::kLanes < 64 ? S::kLanes : 64>(x);
    }
  }
};

struct Args {
  const void* X;
  const void* F;
  const void* dY;
  const void* dH;
  void* Y;
  void* H;
  void* dX;
  void* dF;
  const void* w1;
  const void* b1;
  const void* gate;
  const void* w2;
  const void* b2;
  void* dgate;          // results where a unit is a whole sequence; otherwise units are summed from partial_gate
  float* partial;       // [workgroup][vector][D]: sums over the workgroup's rows of what is wanted of dw1, db1, dgate, dw2, db2
  float* partial_gate;  // [unit][D], gates by sequence
  int layer, D;
  int per_sequence;     // gates
  int take_w1, take_b1, take_gate, take_w2, take_b2, vectors;
  // Rows in units of consecutive ones; with gates by sequence no unit goes over the end of a sequence.
  long long units;
  int unit_rows, sequence_units, sequence_rows;
  float alpha, eps;
  Drop drop;
};

// A unit's rows.
struct Unit {
  long long first, sequence;
  int rows;
  __device__ __forceinline__ Unit(const Args& a, long long unit) {
    sequence = unit / a.sequence_units;
    const int part = static_cast<int>(unit - sequence * a.sequence_units), at = part * a.unit_rows;
    first = sequence * a.sequence_rows + at;
    rows = a.sequence_rows - at < a.unit_rows ? a.sequence_rows - at : a.unit_rows;
  }
};

// What is the same in every row: a lane's columns of the vectors.
template <class T, class S, bool ALIGNED>
struct Columns {
  int col[S::kPieces], valid[S::kPieces];
  __device__ __forceinline__ Columns(int D) {
#pragma unroll
    for (int p = 0; p < S::kPieces; ++p) {
      col[p] = (p * S::kLanes + static_cast<int>(threadIdx.x) % S::kLanes) * 8;
      valid[p] = D - col[p] > 8 ? 8 : D - col[p];
    }
  }
  __device__ __forceinline__ void load(const void* from, long long row, int D, Raw<T> (&to)[S::kPieces]) const {
#pragma unroll
    for (int p = 0; p < S::kPieces; ++p)
      to[p] = residual::load<T, ALIGNED>(static_cast<const T*>(from) + row * D + col[p], valid[p]);
  }
  __device__ __forceinline__ void store(void* to, long long row, int D, int p, const float (&x)[8]) const {
    residual::store<T, ALIGNED>(static_cast<T*>(to) + row * D + col[p], x, valid[p]);
  }
};

// (x - mu) r in place; returns r.  Elements beyond the row are zeros before and after.
template <class S>
__device__ __forceinline__ float normalise(float (&x)[S::kPieces][8], const int (&valid)[S::kPieces], bool layer, float inv_D, float eps,
                                           RowSums<S>& sums) {
  if (layer) {
    float mu = 0.0f;
#pragma unroll
    for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) mu += x[p][i];
    sums(mu);
    mu *= inv_D;
#pragma unroll
    for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[p][i] = i < valid[p] ? x[p][i] - mu : 0.0f;
  }
  float square = 0.0f;
#pragma unroll
  for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) square = fmaf(x[p][i], x[p][i], square);
  sums(square);
  const float r = __builtin_amdgcn_rsqf(fmaf(square, inv_D, eps));
#pragma unroll
  for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[p][i] *= r;
  return r;
}

// A unit's rows one after the other, the next row's on its way.  Bound by memory: 1024 x 200 rows of 256 bf16 (420 MB) in 78 us, 5.4 TB/s;
// fp32 177 us, rows of 1024 ... 8192 as many bytes in 90 ... 95, odd ones of 500, in words that begin anywhere, 173.
template <class T, class S, bool ALIGNED>
__global__ __launch_bounds__(S::kBlock) void seam_fwd_kernel(Args a) {
  __shared__ float lds[S::kWaves > 1 ? 4 * S::kWaves : 1];
  RowSums<S> sums{lds};
  const Columns<T, S, ALIGNED> columns(a.D);
  const Lots lots(a.drop);
  const float inv_D = 1.0f / a.D;
  Raw<T> w1[S::kPieces], b1[S::kPieces], gate[S::kPieces], w2[S::kPieces], b2[S::kPieces];
  if (a.w1 != nullptr) columns.load(a.w1, 0, a.D, w1);
  if (a.b1 != nullptr) columns.load(a.b1, 0, a.D, b1);
  if (a.gate != nullptr && !a.per_sequence) columns.load(a.gate, 0, a.D, gate);
  if (a.w2 != nullptr) columns.load(a.w2, 0, a.D, w2);
  if (a.b2 != nullptr) columns.load(a.b2, 0, a.D, b2);
  for (long long u = static_cast<long long>(blockIdx.x) * S::kGroups + threadIdx.x / S::kLanes; u < a.units;
       u += static_cast<long long>(gridDim.x) * S::kGroups) {
    const Unit unit(a, u);
    if (a.per_sequence) columns.load(a.gate, unit.sequence, a.D, gate);
    Raw<T> rx[S::kPieces], rf[S::kPieces];
    columns.load(a.X, unit.first, a.D, rx);
    columns.load(a.F, unit.first, a.D, rf);
    for (int i = 0; i < unit.rows; ++i) {
      const long long row = unit.first + i;
      float y[S::kPieces][8], f[S::kPieces][8];
#pragma unroll
      for (int p = 0; p < S::kPieces; ++p) {
        unpack<T>(rx[p], y[p]);
        unpack<T>(rf[p], f[p]);
      }
      if (i + 1 < unit.rows) {
        columns.load(a.X, row + 1, a.D, rx);
        columns.load(a.F, row + 1, a.D, rf);
      }
      if (a.w1 != nullptr) normalise<S>(f, columns.valid, a.layer, inv_D, a.eps, sums);
#pragma unroll
      for (int p = 0; p < S::kPieces; ++p) {
        if (a.w1 != nullptr) {
          float w[8], b[8] = {};
          unpack<T>(w1[p], w);
          if (a.b1 != nullptr) unpack<T>(b1[p], b);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[p][e] = fmaf(f[p][e], w[e], b[e]);
        }
        if (a.drop.out_of != 0) {
          const u32x4_t w = lots.template of<ALIGNED>(static_cast<uint64_t>(row) * a.D + columns.col[p]);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[p][e] = lots.keeps(w, e) ? f[p][e] * lots.factor : 0.0f;
        }
        if (a.gate != nullptr) {
          float g[8];
          unpack<T>(gate[p], g);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[p][e] *= g[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[p][e] = fmaf(a.alpha, f[p][e], y[p][e]);
        columns.store(a.Y, row, a.D, p, y[p]);
      }
      if (a.w2 != nullptr) {
        normalise<S>(y, columns.valid, a.layer, inv_D, a.eps, sums);
#pragma unroll
        for (int p = 0; p < S::kPieces; ++p) {
          float w[8], b[8] = {};
          unpack<T>(w2[p], w);
          if (a.b2 != nullptr) unpack<T>(b2[p], b);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[p][e] = fmaf(y[p][e], w[e], b[e]);
          columns.store(a.H, row, a.D, p, y[p]);
        }
      }
    }
  }
}

// d <- r (d - n mean(d n) - mean(d) [layer])
template <class S>
__device__ __forceinline__ void through_norm(float (&d)[S::kPieces][8], const float (&n)[S::kPieces][8], float r, bool layer, float inv_D,
                                             RowSums<S>& sums) {
  float dn = 0.0f, all = 0.0f;
#pragma unroll
  for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dn = fmaf(d[p][e], n[p][e], dn);
      all += d[p][e];
    }
  if (layer) sums(dn, all);
  else sums(dn);
  dn *= inv_D;
  all = layer ? all * inv_D : 0.0f;
#pragma unroll
  for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) d[p][e] = r * (d[p][e] - fmaf(n[p][e], dn, all));
}

template <class S>
__device__ __forceinline__ void clear(float (&x)[S::kPieces][8]) {
#pragma unroll
  for (int p = 0; p < S::kPieces; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[p][e] = 0.0f;
}

// The sums of a workgroup's groups in their order, to its row of a partial vector.
template <class S, bool ALIGNED>
__device__ __forceinline__ void store_partial(float* to, const float (&x)[S::kPieces][8], const int (&col)[S::kPieces],
                                              const int (&valid)[S::kPieces], float* lds) {
  if constexpr (S::kGroups > 1) {
    static_assert(S::kPieces == 1, "rows of a part of a wave are one piece a lane");
    const int group = threadIdx.x / S::kLanes;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[group * S::kMost + e * S::kLanes + threadIdx.x % S::kLanes] = x[0][e];
    __syncthreads();
    for (int at = threadIdx.x; at < S::kMost; at += S::kBlock) {
      float sum = 0.0f;
      for (int g = 0; g < S::kGroups; ++g) sum += lds[g * S::kMost + at];
      lds[at] = sum;  // (in the place of group 0's, which nobody else reads)
    }
    __syncthreads();
    if (group == 0) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = lds[e * S::kLanes + threadIdx.x % S::kLanes];
      store<float, ALIGNED>(to + col[0], y, valid[0]);
    }
  } else {
#pragma unroll
    for (int p = 0; p < S::kPieces; ++p) store<float, ALIGNED>(to + col[p], x[p], valid[p]);
  }
}

// Weights, biases and a gate for all rows as fp32 in LDS, eight values of a lane as two reads that are free of conflicts: held
// in registers they would take those of a second and a third wave.  Rows of more than 2048 elements read them from memory each time.
template <class T, class S, bool ALIGNED>
struct Vectors {
  static constexpr bool kInLds = S::kMost <= 2048;
  static constexpr int kSize = kInLds ? S::kMost : 0;  // floats of one
  const Columns<T, S, ALIGNED>& columns;
  float* at;
  int D;
  __device__ __forceinline__ void set(int slot, const void* from) const {
    if constexpr (kInLds) {
      if (threadIdx.x < S::kLanes && from != nullptr) {
        Raw<T> raw[S::kPieces];
        columns.load(from, 0, D, raw);
        float x[8];
        unpack<T>(raw[0], x);
        f32x4_t* to = reinterpret_cast<f32x4_t*>(at + slot * kSize) + threadIdx.x;
        to[0] = f32x4_t{x[0], x[1], x[2], x[3]};
        to[S::kLanes] = f32x4_t{x[4], x[5], x[6], x[7]};
      }
    }
  }
  __device__ __forceinline__ void get(int slot, const void* from, int p, float (&x)[8]) const {
    if constexpr (kInLds) {
      const f32x4_t* of = reinterpret_cast<const f32x4_t*>(at + slot * kSize) + threadIdx.x % S::kLanes;
      const f32x4_t lo = of[0], hi = of[S::kLanes];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = lo[e];
        x[4 + e] = hi[e];
      }
    } else {
      unpack<T>(residual::load<T, ALIGNED>(static_cast<const T*>(from) + columns.col[p], columns.valid[p]), x);
    }
  }
};

constexpr int max_of(int a, int b) { return a > b ? a : b; }

// Two norms made again and gone through backwards, sums for up to five vectors.
// With the weights in registers and the next row on its way it took 254 registers, one wave a SIMD and 211 us for 1024 x 200 rows of 256 bf16
// (630 MB); with them in LDS, no row ahead and three waves 140, 4.5 TB/s.  fp32 265 us, rows of 1024 151, of 4096 200, of 8192 175, of 500
// in words that begin anywhere 318.  BIAS: the gradient of a bias is wanted.
template <class T, class S, bool ALIGNED, bool BIAS>
__global__ __launch_bounds__(S::kBlock, S::kBlock <= 256 ? 3 : S::kBlock == 512 ? 2 : 4) void seam_bwd_kernel(Args a) {
  typedef Vectors<T, S, ALIGNED> V;
  constexpr int P = S::kPieces;
  enum { kW1, kB1, kGate, kW2 };
  __shared__ __attribute__((aligned(16))) float space[max_of(4 * V::kSize, S::kWaves > 1 ? 4 : S::kGroups * S::kMost)];
  __shared__ float sums_space[S::kWaves > 1 ? 4 * S::kWaves : 1];
  RowSums<S> sums{sums_space};
  const Columns<T, S, ALIGNED> columns(a.D);
  const V vectors{columns, space, a.D};
  const Lots lots(a.drop);
  const float inv_D = 1.0f / a.D;
  vectors.set(kW1, a.w1);
  vectors.set(kB1, a.b1);
  if (!a.per_sequence) vectors.set(kGate, a.gate);
  vectors.set(kW2, a.w2);
  if constexpr (V::kInLds) __syncthreads();
  Raw<T> gate[P];
  float of_w1[P][8], of_b1[BIAS ? P : 1][8], of_gate[P][8], of_w2[P][8], of_b2[BIAS ? P : 1][8];
  clear<S>(of_w1);
  clear<S>(of_gate);
  clear<S>(of_w2);
  if constexpr (BIAS) {
    clear<S>(of_b1);
    clear<S>(of_b2);
  }
  for (long long u = static_cast<long long>(blockIdx.x) * S::kGroups + threadIdx.x / S::kLanes; u < a.units;
       u += static_cast<long long>(gridDim.x) * S::kGroups) {
    const Unit unit(a, u);
    if (a.per_sequence) {
      columns.load(a.gate, unit.sequence, a.D, gate);
      clear<S>(of_gate);
    }
    Raw<T> rx[P], rf[P], ry[P], rh[P];
    auto fetch = [&](long long row) {
      columns.load(a.F, row, a.D, rf);
      if (a.dH != nullptr) {
        columns.load(a.X, row, a.D, rx);
        columns.load(a.dH, row, a.D, rh);
      }
      if (a.dY != nullptr) columns.load(a.dY, row, a.D, ry);
    };
    auto gate_of = [&](int p, float (&g)[8]) {
      if (a.per_sequence) unpack<T>(gate[p], g);
      else vectors.get(kGate, a.gate, p, g);
    };
    for (int i = 0; i < unit.rows; ++i) {
      const long long row = unit.first + i;
      asm volatile("" ::: "memory");  // (what is read from LDS is read again in every row, not held over all)
      fetch(row);
      float f[P][8], z[P][8], d[P][8];
      uint32_t kept[P];
#pragma unroll
      for (int p = 0; p < P; ++p) unpack<T>(rf[p], f[p]);
      float r1 = 0.0f;
      if (a.w1 != nullptr) r1 = normalise<S>(f, columns.valid, a.layer, inv_D, a.eps, sums);
      // z, what the block adds before its gate and alpha
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (a.w1 != nullptr) {
          float w[8], b[8] = {};
          vectors.get(kW1, a.w1, p, w);
          if (a.b1 != nullptr) vectors.get(kB1, a.b1, p, b);
#pragma unroll
          for (int e = 0; e < 8; ++e) z[p][e] = fmaf(f[p][e], w[e], b[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[p][e] = f[p][e];
        }
        kept[p] = 0xffu;
        if (a.drop.out_of != 0) {
          const u32x4_t w = lots.template of<ALIGNED>(static_cast<uint64_t>(row) * a.D + columns.col[p]);
          kept[p] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool keeps = lots.keeps(w, e);
            kept[p] |= keeps ? 1u << e : 0u;
            z[p][e] = keeps ? z[p][e] * lots.factor : 0.0f;
          }
        }
      }
      if (a.dH != nullptr) {
        float y[P][8], h[P][8];
#pragma unroll
        for (int p = 0; p < P; ++p) {
          unpack<T>(rx[p], y[p]);
          unpack<T>(rh[p], h[p]);
          if (a.gate != nullptr) {
            float g[8];
            gate_of(p, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[p][e] = fmaf(a.alpha * g[e], z[p][e], y[p][e]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[p][e] = fmaf(a.alpha, z[p][e], y[p][e]);
          }
        }
        const float r2 = normalise<S>(y, columns.valid, a.layer, inv_D, a.eps, sums);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          float w[8];
          vectors.get(kW2, a.w2, p, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            of_w2[p][e] = fmaf(h[p][e], y[p][e], of_w2[p][e]);
            if constexpr (BIAS) of_b2[p][e] += h[p][e];
            h[p][e] *= w[e];
          }
        }
        through_norm<S>(h, y, r2, a.layer, inv_D, sums);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int e = 0; e < 8; ++e) d[p][e] = (ALIGNED && P == 1) || e < columns.valid[p] ? h[p][e] : 0.0f;
      } else {
        clear<S>(d);
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (a.dY != nullptr) {
          float y[8];
          unpack<T>(ry[p], y);
#pragma unroll
          for (int e = 0; e < 8; ++e) d[p][e] += y[e];
        }
        columns.store(a.dX, row, a.D, p, d[p]);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[p][e] *= a.alpha;
        if (a.gate != nullptr) {
          float g[8];
          gate_of(p, g);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            of_gate[p][e] = fmaf(d[p][e], z[p][e], of_gate[p][e]);
            d[p][e] *= g[e];
          }
        }
        if (a.drop.out_of != 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) d[p][e] = (kept[p] >> e) & 1u ? d[p][e] * lots.factor : 0.0f;
        }
      }
      if (a.w1 != nullptr) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          float w[8];
          vectors.get(kW1, a.w1, p, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            of_w1[p][e] = fmaf(d[p][e], f[p][e], of_w1[p][e]);
            if constexpr (BIAS) of_b1[p][e] += d[p][e];
            d[p][e] *= w[e];
          }
        }
        through_norm<S>(d, f, r1, a.layer, inv_D, sums);
      }
#pragma unroll
      for (int p = 0; p < P; ++p) columns.store(a.dF, row, a.D, p, d[p]);
    }
    if (a.per_sequence && a.take_gate) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (a.sequence_units == 1) columns.store(a.dgate, unit.sequence, a.D, p, of_gate[p]);
        else store<float, ALIGNED>(a.partial_gate + u * a.D + columns.col[p], of_gate[p], columns.valid[p]);
      }
    }
  }
  float* to = a.partial + static_cast<long long>(blockIdx.x) * a.vectors * a.D;
  auto hand_over = [&](bool wanted, const auto& x) {
    if (!wanted) return;
    store_partial<S, ALIGNED>(to, x, columns.col, columns.valid, space);
    to += a.D;
  };
  hand_over(a.take_w1, of_w1);
  if constexpr (BIAS) hand_over(a.take_b1, of_b1);
  hand_over(a.take_gate && !a.per_sequence, of_gate);
  hand_over(a.take_w2, of_w2);
  if constexpr (BIAS) hand_over(a.take_b2, of_b2);
}

// ---- sums over workgroups and units ---------------------------------------------------------------------------------------

struct Sums {
  const float* partial;
  const float* partial_gate;
  void* to[5];
  void* dgate;            // by sequence, or nullptr
  int vectors, blocks, D;
  long long sequences;
  int sequence_units;
  int vector_groups;      // workgroups of the vectors; those of the gates follow
};
constexpr int kSumColumns = 64;                             // of a workgroup
constexpr int kSumWays = 16;                                // that a column's rows are dealt to

// 64 columns a workgroup, 5 us for 768 workgroups' sums of four vectors of 256.  Vectors: sixteen waves sum every sixteenth row, and their sums are joined in order.  Gates by sequence:
// a wave a sequence.
template <class T>
__global__ __launch_bounds__(kSumColumns* kSumWays) void sum_kernel(Sums a) {
  __shared__ float lds[kSumWays][kSumColumns];
  const int lane = threadIdx.x % kSumColumns, way = threadIdx.x / kSumColumns;
  if (static_cast<int>(blockIdx.x) < a.vector_groups) {
    const long long col = static_cast<long long>(blockIdx.x) * kSumColumns + lane, width = static_cast<long long>(a.vectors) * a.D;
    float s = 0.0f;
    if (col < width) {
#pragma unroll 8
      for (int b = way; b < a.blocks; b += kSumWays) s += a.partial[b * width + col];
    }
    lds[way][lane] = s;
    __syncthreads();
    if (way == 0 && col < width) {
#pragma unroll
      for (int w = 1; w < kSumWays; ++w) s += lds[w][lane];
      const int v = static_cast<int>(col / a.D);
      static_cast<T*>(a.to[v])[col - static_cast<long long>(v) * a.D] = static_cast<T>(s);
    }
  } else {
    const int column_groups = (a.D + kSumColumns - 1) / kSumColumns;
    const long long at = blockIdx.x - a.vector_groups;
    const long long sequence = at / column_groups * kSumWays + way;
    const int col = static_cast<int>(at % column_groups) * kSumColumns + lane;
    if (sequence >= a.sequences || col >= a.D) return;
    const float* p = a.partial_gate + sequence * a.sequence_units * a.D + col;
    float s = 0.0f;
#pragma unroll 8
    for (int u = 0; u < a.sequence_units; ++u) s += p[static_cast<long long>(u) * a.D];
    static_cast<T*>(a.dgate)[sequence * a.D + col] = static_cast<T>(s);
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------------

constexpr int kMostWidth = 8192;

// Lanes of a row: as few as take it in one piece of eight each, which leaves the sums over the row short and several rows to a wave.
int lanes_of(int D) { return D <= 64 ? 8 : D <= 256 ? 32 : D <= 512 ? 64 : D <= 1024 ? 128 : D <= 2048 ? 256 : D <= 4096 ? 512 : 1024; }

struct Plan {
  long long units, sequences;
  int unit_rows, sequence_units, sequence_rows, blocks;
  // `rows` of `sequence_rows` each where gates go by sequence; otherwise all rows count as one sequence, cut so that rows
  // numbered with 31 bits are enough (the last sequence may be shorter: then there is only one).
  Plan(int B, int N, int D, bool per_sequence, bool bwd) {
    const int lanes = lanes_of(D), block = lanes > 64 ? lanes : kThreads, groups = block / lanes;
    // as many workgroups as run at once: 1024 threads to a compute unit, or 768 where the backward's registers admit no more
    const int at_once = bwd && block <= 256 ? 768 / block : bwd ? 1 : 1024 / block;
    const long long most_groups = 256ll * at_once * groups;
    const long long rows = static_cast<long long>(B) * N;
    sequences = per_sequence ? B : 1;
    sequence_rows = per_sequence ? N : static_cast<int>(rows);
    const long long per_group = (rows + most_groups - 1) / most_groups;
    long long parts = (sequence_rows + per_group - 1) / per_group;
    unit_rows = static_cast<int>((sequence_rows + parts - 1) / parts);
    sequence_units = (sequence_rows + unit_rows - 1) / unit_rows;
    units = sequences * sequence_units;
    const long long wanted = (units + groups - 1) / groups, most = most_groups / groups;
    blocks = static_cast<int>(wanted < most ? wanted : most);
  }
};

template <class T, bool ALIGNED>
void launch_seam(const Args& a, int blocks, bool bwd, hipStream_t s) {
#define COTTEN_SEAM(LANES)                                                                                    \
  {                                                                                                           \
    typedef Shape<LANES> S;                                                                                   \
    const dim3 grid(blocks), block(S::kBlock);                                                                \
    if (!bwd) seam_fwd_kernel<T, S, ALIGNED><<<grid, block, 0, s>>>(a);                                       \
    else if (a.take_b1 || a.take_b2) seam_bwd_kernel<T, S, ALIGNED, true><<<grid, block, 0, s>>>(a);          \
    else seam_bwd_kernel<T, S, ALIGNED, false><<<grid, block, 0, s>>>(a);                                     \
  }
  const int D = a.D;
  if (D <= 64) COTTEN_SEAM(8)
  else if (D <= 256) COTTEN_SEAM(32)
  else if (D <= 512) COTTEN_SEAM(64)
  else if (D <= 1024) COTTEN_SEAM(128)
  else if (D <= 2048) COTTEN_SEAM(256)
  else if (D <= 4096) COTTEN_SEAM(512)
  else COTTEN_SEAM(1024)
#undef COTTEN_SEAM
}

template <class T>
hipError_t launch(const Args& a, const Plan& plan, bool bwd, hipStream_t s) {
  if (a.D % 8 == 0) launch_seam<T, true>(a, plan.blocks, bwd, s);
  else launch_seam<T, false>(a, plan.blocks, bwd, s);
  return hipGetLastError();
}

template <class T>
hipError_t launch_sums(const Sums& a, long long groups, hipStream_t s) {
  sum_kernel<T><<<dim3(static_cast<unsigned>(groups)), dim3(kSumColumns * kSumWays), 0, s>>>(a);
  return hipGetLastError();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_drop(Drop* d, double p, uint64_t seed, uint64_t offset, const int64_t* step) {
  if (!(p >= 0.0 && p < 1.0)) return COTTEN_ERR_BAD_PARAM;
  const double out_of = std::floor(p * 65536.0 + 0.5);
  if (out_of > 65535.0) return COTTEN_ERR_BAD_PARAM;
  if (reinterpret_cast<uintptr_t>(step) & 7u) return COTTEN_ERR_MISALIGNED;
  d->seed = seed;
  d->offset = offset;
  d->step = reinterpret_cast<const long long*>(step);
  d->out_of = static_cast<uint32_t>(out_of);
  d->factor = static_cast<float>(65536.0 / (65536.0 - out_of));
  return COTTEN_OK;
}

int check_shape(int B, int N, int D) {
  if (B < 1 || N < 1 || D < 1 || D > kMostWidth || static_cast<long long>(B) * N >= (1ll << 31)) return COTTEN_ERR_BAD_SHAPE;
  return COTTEN_OK;
}

// What both directions share.
int prepare(Args* a, const void* X, const void* F, int B, int N, int D, const cotten_residual_params* prm) {
  if (prm == nullptr || X == nullptr || F == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (prm->dtype != COTTEN_F32 && prm->dtype != COTTEN_BF16 && prm->dtype != COTTEN_F16) return COTTEN_ERR_BAD_DTYPE;
  if (int rc = check_shape(B, N, D)) return rc;
  if (prm->norm != COTTEN_NORM_RMS && prm->norm != COTTEN_NORM_LAYER) return COTTEN_ERR_BAD_PARAM;
  if ((prm->post_bias != nullptr && prm->post_weight == nullptr) || (prm->next_bias != nullptr && prm->next_weight == nullptr))
    return COTTEN_ERR_BAD_PARAM;
  if (!std::isfinite(prm->alpha) || !std::isfinite(prm->eps)) return COTTEN_ERR_BAD_PARAM;
  if (int rc = check_drop(&a->drop, prm->p, prm->seed, prm->offset, prm->step)) return rc;
  const void* tensors[] = {X, F, prm->post_weight, prm->post_bias, prm->gate, prm->next_weight, prm->next_bias, prm->workspace};
  for (const void* t : tensors)
    if (!aligned16(t)) return COTTEN_ERR_MISALIGNED;
  a->X = X;
  a->F = F;
  a->w1 = prm->post_weight;
  a->b1 = prm->post_bias;
  a->gate = prm->gate;
  a->w2 = prm->next_weight;
  a->b2 = prm->next_bias;
  a->layer = prm->norm == COTTEN_NORM_LAYER;
  a->per_sequence = prm->gate != nullptr && prm->gate_per_sequence;
  a->D = D;
  a->alpha = prm->alpha;
  a->eps = prm->eps < 0.0f ? 1e-6f : prm->eps;
  return COTTEN_OK;
}

void use_plan(Args* a, const Plan& plan) {
  a->units = plan.units;
  a->unit_rows = plan.unit_rows;
  a->sequence_units = plan.sequence_units;
  a->sequence_rows = plan.sequence_rows;
}

hipError_t launch_any(int dtype, const Args& a, const Plan& plan, bool bwd, hipStream_t s) {
  return dtype == COTTEN_F32 ? launch<float>(a, plan, bwd, s)
         : dtype == COTTEN_BF16 ? launch<__bf16>(a, plan, bwd, s)
                                : launch<_Float16>(a, plan, bwd, s);
}

}  // namespace
}  // namespace residual
}  // namespace cotten

using namespace cotten::residual;

extern "C" {

int cotten_dropout(const void* x, void* y, size_t n, void* stream, const cotten_dropout_params* prm) {
  if (prm == nullptr || x == nullptr || y == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (prm->dtype != COTTEN_F32 && prm->dtype != COTTEN_BF16 && prm->dtype != COTTEN_F16) return COTTEN_ERR_BAD_DTYPE;
  if (n < 1 || n >= (1ull << 40)) return COTTEN_ERR_BAD_SHAPE;
  cotten::Drop drop;
  if (int rc = check_drop(&drop, prm->p, prm->seed, prm->offset, prm->step)) return rc;
  if (!aligned16(x) || !aligned16(y)) return COTTEN_ERR_MISALIGNED;
  const size_t pieces = (n + 7) / 8, of_block = kThreads * kDropPieces;
  const size_t wanted = (pieces + of_block - 1) / of_block;
  const dim3 grid(static_cast<unsigned>(wanted < (1u << 20) ? wanted : (1u << 20))), block(kThreads);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (prm->dtype == COTTEN_F32) dropout_kernel<float><<<grid, block, 0, s>>>(static_cast<const float*>(x), static_cast<float*>(y), n, drop);
  else if (prm->dtype == COTTEN_BF16) dropout_kernel<__bf16><<<grid, block, 0, s>>>(static_cast<const __bf16*>(x), static_cast<__bf16*>(y), n, drop);
  else dropout_kernel<_Float16><<<grid, block, 0, s>>>(static_cast<const _Float16*>(x), static_cast<_Float16*>(y), n, drop);
  return hipGetLastError() == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

size_t cotten_residual_workspace_bytes(int B, int N, int D, int gate_per_sequence) {
  if (check_shape(B, N, D) != COTTEN_OK) return 0;
  const Plan plan(B, N, D, gate_per_sequence != 0, true);
  return (static_cast<size_t>(plan.blocks) * 5 + (gate_per_sequence && plan.sequence_units > 1 ? plan.units : 0)) * D * sizeof(float);
}

int cotten_residual_fwd(const void* X, const void* F, void* Y, void* H, int B, int N, int D, void* stream,
                        const cotten_residual_params* prm) {
  Args a{};
  if (int rc = prepare(&a, X, F, B, N, D, prm)) return rc;
  if (Y == nullptr || (H == nullptr) != (prm->next_weight == nullptr)) return COTTEN_ERR_NULL_POINTER;
  if (!aligned16(Y) || !aligned16(H)) return COTTEN_ERR_MISALIGNED;
  a.Y = Y;
  a.H = H;
  const Plan plan(B, N, D, a.per_sequence, false);
  use_plan(&a, plan);
  return launch_any(prm->dtype, a, plan, false, static_cast<hipStream_t>(stream)) == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

int cotten_residual_bwd(const void* X, const void* F, const void* dY, const void* dH, void* dX, void* dF, int B, int N, int D,
                        void* stream, const cotten_residual_params* prm, const cotten_residual_grads* grads) {
  Args a{};
  if (int rc = prepare(&a, X, F, B, N, D, prm)) return rc;
  if (dX == nullptr || dF == nullptr || grads == nullptr || (dY == nullptr && dH == nullptr)) return COTTEN_ERR_NULL_POINTER;
  if (dH != nullptr && prm->next_weight == nullptr) return COTTEN_ERR_BAD_PARAM;
  struct { void* to; const void* of; } pairs[] = {{grads->post_weight, prm->post_weight}, {grads->post_bias, prm->post_bias},
                                                  {grads->gate, prm->gate}, {grads->next_weight, prm->next_weight},
                                                  {grads->next_bias, prm->next_bias}};
  for (const auto& p : pairs) {
    if (p.to != nullptr && p.of == nullptr) return COTTEN_ERR_BAD_PARAM;
    if (!aligned16(p.to)) return COTTEN_ERR_MISALIGNED;
  }
  if (!aligned16(dY) || !aligned16(dH) || !aligned16(dX) || !aligned16(dF)) return COTTEN_ERR_MISALIGNED;
  const Plan plan(B, N, D, a.per_sequence, true);
  use_plan(&a, plan);
  if (prm->workspace == nullptr ||
      prm->workspace_bytes < cotten_residual_workspace_bytes(B, N, D, a.per_sequence)) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  a.dY = dY;
  a.dH = dH;
  a.dX = dX;
  a.dF = dF;
  a.dgate = grads->gate;
  a.partial = static_cast<float*>(prm->workspace);
  a.partial_gate = a.partial + static_cast<size_t>(plan.blocks) * 5 * D;
  a.take_w1 = grads->post_weight != nullptr;
  a.take_b1 = grads->post_bias != nullptr;
  a.take_gate = grads->gate != nullptr;
  a.take_w2 = grads->next_weight != nullptr;
  a.take_b2 = grads->next_bias != nullptr;
  Sums sums{};
  void* const to[5] = {grads->post_weight, grads->post_bias, a.per_sequence ? nullptr : grads->gate, grads->next_weight, grads->next_bias};
  for (void* t : to)
    if (t != nullptr) sums.to[a.vectors++] = t;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (launch_any(prm->dtype, a, plan, true, s) != hipSuccess) return COTTEN_ERR_LAUNCH;
  sums.partial = a.partial;
  sums.partial_gate = a.partial_gate;
  sums.vectors = a.vectors;
  sums.blocks = plan.blocks;
  sums.D = D;
  sums.sequences = plan.sequences;
  sums.sequence_units = plan.sequence_units;
  sums.vector_groups = static_cast<int>((static_cast<long long>(a.vectors) * D + kSumColumns - 1) / kSumColumns);
  long long groups = sums.vector_groups;
  if (a.per_sequence && a.take_gate && plan.sequence_units > 1) {
    sums.dgate = grads->gate;
    groups += (plan.sequences + kSumWays - 1) / kSumWays * ((D + kSumColumns - 1) / kSumColumns);
  }
  if (groups == 0) return COTTEN_OK;
  const hipError_t rc = prm->dtype == COTTEN_F32    ? launch_sums<float>(sums, groups, s)
                        : prm->dtype == COTTEN_BF16 ? launch_sums<__bf16>(sums, groups, s)
                                                    : launch_sums<_Float16>(sums, groups, s);
  return rc == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

}  // extern "C"
