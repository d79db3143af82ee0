// Device code of the decay attention: linear attention on unit rows with one decay for each head.  With x^ = x / sqrt(|x|^2 + eps),
// a = exp(g of the head) and, for a masked token, S_t = S_{t-1}:
//
//     S_t = a S_{t-1} + k^_t v_t^T          o_t = scale * S_t^T q^_t
//
// Over a chunk of 32 tokens, with p_t how many of them up to t count (n of the whole chunk) and S the state before it:
//
//     O_i = scale (sum_{j <= i} a^(p_i - p_j) (q^_i . k^_j) v_j + a^(p_i) S^T q^_i)      S' = a^n S + sum_j a^(n - p_j) k^_j v_j^T
//
// The gradients have the same form, with other rows in the places of queries, keys and values, from the first chunk to the last or
// back (dS after the chunk, dS' before it):
//
//     dq^_i = scale (sum_{j <= i} a^(p_i - p_j) (dO_i . v_j) k^_j + a^(p_i) S dO_i)
//     dk^_j = sum_{i >= j} a^(p_i - p_j) scale (v_j . dO_i) q^_i + a^(n - p_j) dS v_j
//     dv_j  = sum_{i >= j} a^(p_i - p_j) scale (k^_j . q^_i) dO_i + a^(n - p_j) dS^T k^_j       dS' = a^n dS + sum_i a^(p_i) scale q^_i dO_i^T
//
// so one walk serves all: rows X (what a result row belongs to), Y and Z (what it is summed over), a state of Y^T Z, and a
// factor of each row of X and of each pair of rows Y and Z, which take norms, scale and decays.  The norms' Jacobian,
// dq = (dq^ - q^ (q^ . dq^)) / r(q), is an epilogue.  The decays' gradient is that of the outputs by g, which carries T = dS_t / dg too:
//
//     dg = sum_i dO_i . (scale (sum_{j <= i} (p_i - p_j) a^(p_i - p_j) (q^_i . k^_j) v_j + a^(p_i) (p_i S + T)^T q^_i)) + <dS_N, T_N>
//     T' = a^n (T + n S) + sum_j (n - p_j) a^(n - p_j) k^_j v_j^T
//
// with no sums that cancel, however strong the decay.
//
// Precision.  As in the gated delta rule operands are cut into bf16 pieces and products keep those that reach 24 bits: states leave in fp32.
// a^n multiplies the state once a chunk, the same factor each time: it is kept as two floats, or its rounding would add up
// over the thousands of chunks that a weak decay spans.
#pragma once
#include "cotten_delta_chunk.h"

namespace cotten {
namespace decay {

using delta::buffer;
using delta::cut;
using delta::existing;
using delta::f32x4_t;
using delta::kChunk;
using delta::kNowhere;
using delta::lds_barrier;
using delta::mul;
using delta::mul_left;
using delta::mul_right;
using delta::offset_if;
using delta::over_groups;
using delta::Pieces;
using delta::Rows;
using delta::StateColumns;

struct Args {
  const unsigned char* Q;
  const unsigned char* K;
  const unsigned char* V;
  const unsigned char* dO;
  const float* g;               // [H]
  const uint8_t* mask;          // [B,N] or nullptr
  unsigned char* O;
  unsigned char* dQ;
  unsigned char* dK;
  unsigned char* dV;
  const float* initial_state;   // [B*H][D][D] or nullptr
  float* final_state;
  const float* dfinal_state;
  float* dinitial_state;
  // Sequences cut into segments: what a segment alone adds to the state behind it, to its derivative by g and to the gradient
  // of the state before it, and how many of its tokens count.
  float* local_s;               // [slice][segment][D][D]; the last one's place holds a copy of the initial state (forward)
  float* local_t;
  float* local_d;
  float* counts;                // [slice][segment]
  double* dg;                   // [slice][segment][part]: partial sums of the decays' gradient
  int segments, segment_chunks;
  int H, N, chunks;
  long long stride_batch, stride_head;  // in bytes
  uint32_t stride_row;
  float scale, eps;
};

// What a walk makes.  kStates and kGradStates: a segment's local states alone.
enum Role { kOut, kDq, kDk, kDv, kDecays, kStates, kStatesAndDerivatives, kGradStates };

template <int ROLE>
struct Traits {
  static constexpr bool kBack = ROLE == kDk || ROLE == kDv || ROLE == kGradStates;       // from the last chunk to the first
  static constexpr bool kRows = ROLE < kStates;                                         // makes rows, not only a state
  static constexpr bool kThrough = ROLE == kDq || ROLE == kDk;                          // through the norm of a row
  static constexpr bool kDerivative = ROLE == kDecays || ROLE == kStatesAndDerivatives; // carries T
  static constexpr bool kTransposed = ROLE == kDq || ROLE == kDk;                       // its state is S^T or dS^T
  // the tensors in the places of X, Y, Z
  static __device__ __forceinline__ const unsigned char* x(const Args& a) {
    return ROLE == kDq ? a.dO : ROLE == kDk ? a.V : ROLE == kDv ? a.K : a.Q;
  }
  static __device__ __forceinline__ const unsigned char* y(const Args& a) {
    return ROLE == kDq ? a.V : ROLE == kDk ? a.dO : kBack ? a.Q : a.K;
  }
  static __device__ __forceinline__ const unsigned char* z(const Args& a) {
    return ROLE == kDq ? a.K : ROLE == kDk ? a.Q : kBack ? a.dO : a.V;
  }
  // which of them are unit rows, and which the scale goes with
  static constexpr bool kUnitX = ROLE == kOut || ROLE == kDecays || ROLE == kDv;
  static constexpr bool kUnitY = ROLE != kDq && ROLE != kDk;
  static constexpr bool kUnitZ = !kUnitY;
  static constexpr bool kScaleX = !kBack;
};

// What a wave knows of its slice.
struct Slice {
  long long rows;
  const uint8_t* mask;
  uint32_t bytes;
  float g;
  __device__ __forceinline__ Slice(const Args& a, int slice, uint32_t row_bytes) {
    const int b = slice / a.H, h = slice - b * a.H;
    rows = b * a.stride_batch + h * a.stride_head;
    mask = a.mask == nullptr ? nullptr : a.mask + static_cast<long long>(b) * a.N;
    bytes = static_cast<uint32_t>(a.N - 1) * a.stride_row + row_bytes;
    g = a.g[h];
  }
  // from a chunk's first row on; rows beyond the sequence are beyond the buffer
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t of(const unsigned char* base, int chunk, uint32_t stride) const {
    const uint32_t skip = static_cast<uint32_t>(kChunk * chunk) * stride;
    return buffer(base + rows + skip, skip < bytes ? bytes - skip : 0);
  }
};

// The tokens of a chunk that count, a bit each; the bytes are asked for a chunk ahead.
struct Mask {
  __amdgpu_buffer_rsrc_t bytes;
  bool all;
  int N;
  uint32_t byte = 0;
  __device__ __forceinline__ Mask(const Args& a, const Slice& s) : bytes(buffer(s.mask, s.mask == nullptr ? 0 : a.N)), all(s.mask == nullptr), N(a.N) {}
  __device__ __forceinline__ void fetch(int chunk, int lane) {
    byte = __builtin_amdgcn_raw_buffer_load_b8(bytes, chunk < 0 ? kNowhere : static_cast<uint32_t>(kChunk * chunk + (lane & 31)), 0, 0);
  }
  __device__ __forceinline__ uint32_t bits(int chunk) const { return all ? existing(N, chunk) : static_cast<uint32_t>(__ballot(byte != 0)); }
};

// g * log2(e) as two floats.  A decay to nothing (g = -inf) counts as 2^-100000: fp32 knows no difference, and no tokens are none.
struct Rate {
  float hi, lo;
  double whole;
  __device__ __forceinline__ explicit Rate(float g) {
    whole = static_cast<double>(g) * 1.4426950408889634;
    whole = whole < -100000.0 ? -100000.0 : whole;
    hi = static_cast<float>(whole);
    lo = static_cast<float>(whole - hi);
  }
  // a^n, n a small whole number
  __device__ __forceinline__ float pow(float n) const {
    const float x = n * hi, rest = fmaf(n, hi, -x) + n * lo, e = __builtin_amdgcn_exp2f(x);
    return fmaf(e * 0.693147182f, rest, e);
  }
};

// Counts of the tokens of a chunk, and the factors that follow from them, for a lane's tokens: column 16 t + lane%16, rows 16 t + 4g + r.
// They are the same in all chunks whose tokens all count.
template <class R>
struct Decays {
  uint32_t live;
  float n;                  // tokens that count
  float to[2];              // of X's rows, against the state
  float column[2];          // p of them
  float fro[2][4];          // of Z's rows, for the state
  float row[2][4];          // p of these
  float pair[3][4];         // of the pairs of tile 0 with 0, of X tile 0 with Y tile 1 (back) or 1 with 0, of 1 with 1
  float whole_hi, whole_lo;
  static __device__ __forceinline__ float upto(uint32_t live, int t) { return static_cast<float>(__popc(live & (0xffffffffu >> (31 - t)))); }
  __device__ __forceinline__ void set(uint32_t bits, const Rate& rate, int lane) {
    live = bits;
    const int c = lane & 15, first = 4 * (lane >> 4);
    n = static_cast<float>(__popc(bits));
    const double w = exp2(rate.whole * static_cast<double>(n));
    whole_hi = static_cast<float>(w);
    whole_lo = static_cast<float>(w - static_cast<double>(whole_hi));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      column[t] = upto(bits, 16 * t + c);
      to[t] = rate.pow(R::kBack ? n - column[t] : column[t]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        row[t][r] = upto(bits, 16 * t + first + r);
        fro[t][r] = rate.pow(R::kBack ? row[t][r] : n - row[t][r]);
      }
    }
    if constexpr (R::kRows) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool in = R::kBack ? first + r >= c : first + r <= c;
        pair[0][r] = in ? rate.pow(apart(0, 0, r)) : 0.0f;
        pair[1][r] = R::kBack ? rate.pow(apart(0, 1, r)) : rate.pow(apart(1, 0, r));
        pair[2][r] = in ? rate.pow(apart(1, 1, r)) : 0.0f;
      }
    }
  }
  // tokens that count between column 16 x + lane%16 and row 16 y + 4g + r
  __device__ __forceinline__ float apart(int x, int y, int r) const { return R::kBack ? row[y][r] - column[x] : column[x] - row[y][r]; }
};

// x by columns as they lie in a state: 16 dt + 4g + r of row `col`.
template <int D>
__device__ __forceinline__ void load_transposed(StateColumns<D>& S, const float* from, int col, int lane) {
  const __amdgpu_buffer_rsrc_t r = StateColumns<D>::of(from);
#pragma unroll
  for (int dt = 0; dt < 2 * StateColumns<D>::kBlocks; ++dt)
    S.s[dt] = dt < StateColumns<D>::kTiles
                  ? __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, (col * D + 16 * dt + 4 * (lane >> 4)) * 4, 0, 0))
                  : f32x4_t{0, 0, 0, 0};
}
template <int D, bool TRANSPOSED>
__device__ __forceinline__ void load_state(StateColumns<D>& S, const float* from, int col, int lane) {
  if constexpr (TRANSPOSED) load_transposed<D>(S, from, col, lane);
  else S.load(from, col, lane);
}

template <int D>
constexpr int kWaves = D / 16;

// A chunk's place in LDS: rows in pieces, and the factors of X's rows and of the pairs of Y's and Z's.
template <class E, int D, bool ROWS>
struct Place {
  typedef Rows<D, E::kPieces> R;
  static constexpr int kY = 0, kZ = R::kBytes, kX = 2 * R::kBytes, kOfX = ROWS ? 3 * R::kBytes : 2 * R::kBytes;
  static constexpr int kOfPair = kOfX + kChunk * 4, kBytes = kOfPair + kChunk * 4;
};
template <class E, int D, int ROLE>
constexpr int kLds = Place<E, D, Traits<ROLE>::kRows>::kBytes + (Traits<ROLE>::kThrough ? kWaves<D> * kChunk * 8 : 64);

// Sum over the LANES lanes that share a row, in all of them.
template <int LANES>
__device__ __forceinline__ float over_row(float x) {
  if constexpr (LANES > 1) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), 0xB1, 0xF, 0xF, true));
  if constexpr (LANES > 2) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), 0x4E, 0xF, 0xF, true));
  if constexpr (LANES > 4) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), 0x141, 0xF, 0xF, true));
  if constexpr (LANES > 8) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), 0x140, 0xF, 0xF, true));
  return x;
}
template <class E, int D>
__device__ __forceinline__ float inverse_norm(const typename E::Raw& raw, float eps) {
  float x[8], s = 0.0f;
  E::unpack(raw, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
  return __builtin_amdgcn_rsqf(over_row<D / 8>(s) + eps);
}

// Four columns of two rows (tokens lane%16 and 16 more) of a result, or of the rows it belongs to.
template <class E>
struct ResultRows {
  f32x4_t x[2];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t stride, uint32_t live, uint32_t first, int lane) {
#pragma unroll
    for (int t = 0; t < 2; ++t) x[t] = E::load_four(r, offset_if(live, 16 * t + (lane & 15), first + 16 * t * stride));
  }
};

// The walk of one unit: a slice, or a segment of it.  Every wave carries 16 columns of the state; all load the chunk's rows (a wave 512 / D of
// each tensor, eight elements a lane) and leave them in LDS in pieces.
template <class E, int D, int ROLE>
__device__ void walk(const Args& a, int unit, unsigned char* smem) {
  typedef Traits<ROLE> R;
  typedef Place<E, D, R::kRows> P;
  typedef typename P::R L;
  constexpr int kRowLanes = D / 8, kBlocks = StateColumns<D>::kBlocks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slice = unit / a.segments, segment = unit - slice * a.segments;
  const Slice s(a, slice, D * E::kBytes);
  const Rate rate(s.g);
  const int begin = segment * a.segment_chunks;
  const int end = begin + a.segment_chunks < a.chunks ? begin + a.segment_chunks : a.chunks;
  const int col = 16 * wave + (lane & 15), group = lane >> 4;
  const long long of_slice = static_cast<long long>(slice) * a.segments;
  const long long state_at = static_cast<long long>(slice) * D * D;
  float* of_x = reinterpret_cast<float*>(smem + P::kOfX);
  float* of_pair = reinterpret_cast<float*>(smem + P::kOfPair);

  if (D < 32) {  // narrow rows are followed by zeros
    for (int i = threadIdx.x; i < P::kOfX / 16; i += 64 * kWaves<D>) reinterpret_cast<f32x4_t*>(smem)[i] = f32x4_t{0, 0, 0, 0};
    lds_barrier();
  }

  // the state before the first chunk (back: behind the last)
  StateColumns<D> S, T;
  const float* outer = R::kBack ? a.dfinal_state : a.initial_state;
  outer = outer == nullptr ? nullptr : outer + state_at;
  if constexpr (R::kDerivative) load_state<D, false>(T, nullptr, col, lane);
  if constexpr (!R::kRows) {
    // the outermost segment's local state holds what comes from outside
    const bool outermost = R::kBack ? segment == a.segments - 1 : segment == 0;
    load_state<D, false>(S, outermost ? outer : nullptr, col, lane);
    if (!R::kBack && segment == a.segments - 1) {
      // nobody needs this one's: its place takes a copy of the initial state, which the segments' walks start from (final_state may be
      // initial_state, and another workgroup writes it)
      load_state<D, false>(S, outer, col, lane);
      S.store(a.local_s + (of_slice + segment) * D * D, col, lane);
      return;
    }
    if (R::kBack && segment == 0) return;
  } else if (a.segments == 1) {
    load_state<D, R::kTransposed>(S, outer, col, lane);
  } else if (R::kBack) {
    if (segment == a.segments - 1) {
      load_state<D, R::kTransposed>(S, outer, col, lane);
    } else {
      load_state<D, R::kTransposed>(S, a.local_d + (of_slice + a.segments - 1) * D * D, col, lane);
      for (int j = a.segments - 2; j > segment; --j) {
        const float w = static_cast<float>(exp2(rate.whole * static_cast<double>(a.counts[of_slice + j])));
        load_state<D, R::kTransposed>(T, a.local_d + (of_slice + j) * D * D, col, lane);
#pragma unroll
        for (int dt = 0; dt < 2 * kBlocks; ++dt) S.s[dt] = S.s[dt] * w + T.s[dt];
      }
    }
  } else {
    load_state<D, R::kTransposed>(S, a.local_s + (of_slice + (segment == 0 ? a.segments - 1 : 0)) * D * D, col, lane);
    if constexpr (R::kDerivative)
      if (segment > 0) load_state<D, false>(T, a.local_t + of_slice * D * D, col, lane);
    for (int j = 1; j < segment; ++j) {
      const float n = a.counts[of_slice + j], w = static_cast<float>(exp2(rate.whole * static_cast<double>(n)));
      if constexpr (R::kDerivative) {
        StateColumns<D> next;
        load_state<D, false>(next, a.local_t + (of_slice + j) * D * D, col, lane);
#pragma unroll
        for (int dt = 0; dt < 2 * kBlocks; ++dt) T.s[dt] = w * (T.s[dt] + n * S.s[dt]) + next.s[dt];
      }
      StateColumns<D> next;
      load_state<D, R::kTransposed>(next, a.local_s + (of_slice + j) * D * D, col, lane);
#pragma unroll
      for (int dt = 0; dt < 2 * kBlocks; ++dt) S.s[dt] = S.s[dt] * w + next.s[dt];
    }
  }

  Mask mask(a, s);
  uint32_t live, there;
  typename E::Raw rx, ry, rz;
  ResultRows<E> own;                        // rows of Q or K (through their norm), or of dO (decays)
  const int row = wave * (512 / D) + lane / kRowLanes;
  const uint32_t off = static_cast<uint32_t>(row) * a.stride_row + (lane % kRowLanes) * 8 * E::kBytes;
  const uint32_t own_off = static_cast<uint32_t>(lane & 15) * a.stride_row + (16 * wave + 4 * group) * E::kBytes;
  auto fetch = [&](int chunk) {
    live = mask.bits(chunk);
    there = existing(a.N, chunk);
    // forwards the mask is that of Y and Z, back that of X
    const uint32_t at_x = R::kBack ? offset_if(live, row, off) : off, at_yz = R::kBack ? off : offset_if(live, row, off);
    if constexpr (R::kRows) rx = E::load(s.of(R::x(a), chunk, a.stride_row), at_x);
    ry = E::load(s.of(R::y(a), chunk, a.stride_row), at_yz);
    rz = E::load(s.of(R::z(a), chunk, a.stride_row), at_yz);
  };
  const int step = R::kBack ? -1 : 1, first = R::kBack ? end - 1 : begin, last = R::kBack ? begin : end - 1;
  mask.fetch(first, lane);
  fetch(first);
  if (first != last) mask.fetch(first + step, lane);

  Decays<R> decays;
  decays.set(live, rate, lane);
  float count = 0.0f;
  double sum = 0.0;
  f32x4_t held[2];                          // rows that wait for the sums over the waves
  uint32_t held_live = 0;
  float* parts = reinterpret_cast<float*>(smem + P::kBytes);   // [wave][token]: y . x^ and y . y
  auto finish = [&](int chunk) {
    unsigned char* to = ROLE == kDq ? a.dQ : a.dK;
    const __amdgpu_buffer_rsrc_t r = s.of(to, chunk, a.stride_row);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int token = 16 * t + (lane & 15);
      float dot = 0.0f, square = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves<D>; ++w) {
        dot += parts[(w * kChunk + token) * 2];
        square += parts[(w * kChunk + token) * 2 + 1];
      }
      const float inverse = __builtin_amdgcn_rsqf(square + a.eps), back = dot * inverse * inverse;
      f32x4_t x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = ((held_live >> token) & 1u) ? inverse * (held[t][i] - own.x[t][i] * back) : 0.0f;
      E::store_four(r, own_off + 16 * t * a.stride_row, x);
    }
  };

  for (int c = first;; c += step) {
    // rows to LDS
    const uint32_t now = live, now_there = there;
    const int of_row = wave * (512 / D) + lane / kRowLanes;
    {
      const int kb = (lane % kRowLanes) / 4, g = (lane % kRowLanes) % 4;
      float fx = 1.0f, fyz = 1.0f;
      if constexpr (R::kRows) {
        L::put(smem + P::kX, of_row, kb, g, E::pieces(rx));
        if constexpr (R::kUnitX) fx = inverse_norm<E, D>(rx, a.eps);
      }
      L::put(smem + P::kY, of_row, kb, g, E::pieces(ry));
      L::put(smem + P::kZ, of_row, kb, g, E::pieces(rz));
      fyz = inverse_norm<E, D>(R::kUnitY ? ry : rz, a.eps);
      if (R::kScaleX) fx *= a.scale;
      else fyz *= a.scale;
      const uint32_t in_x = R::kBack ? now : now_there, in_yz = R::kBack ? now_there : now;
      if (lane % kRowLanes == 0) {
        of_x[of_row] = ((in_x >> of_row) & 1u) ? fx : 0.0f;
        of_pair[of_row] = ((in_yz >> of_row) & 1u) ? fyz : 0.0f;
      }
    }
    if (now != decays.live) decays.set(now, rate, lane);
    if (c != last) {
      fetch(c + step);
      if (c + step != last) mask.fetch(c + 2 * step, lane);
    }
    lds_barrier();

    const f32x4_t pair_factor[2] = {*reinterpret_cast<const f32x4_t*>(of_pair + 4 * group), *reinterpret_cast<const f32x4_t*>(of_pair + 16 + 4 * group)};
    const Pieces<E::kPieces> z = L::column_operand(smem + P::kZ, wave, lane);
    if constexpr (R::kRows) {
      const float x_factor[2] = {of_x[lane & 15], of_x[16 + (lane & 15)]};
      if constexpr (R::kThrough || ROLE == kDecays)
        own.load(s.of(ROLE == kDq ? a.Q : ROLE == kDk ? a.K : a.dO, c, a.stride_row), a.stride_row, R::kBack ? now : ~0u, own_off, lane);
      // the products of X's rows with Y's: rows Y, columns X
      Pieces<E::kPieces> x[2][kBlocks];
      f32x4_t d[3] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) {
        const Pieces<E::kPieces> y[2] = {L::row_operand(smem + P::kY, 0, kb, lane), L::row_operand(smem + P::kY, 1, kb, lane)};
        x[0][kb] = L::row_operand(smem + P::kX, 0, kb, lane);
        x[1][kb] = L::row_operand(smem + P::kX, 1, kb, lane);
        d[0] = mul(y[0], x[0][kb], d[0]);
        d[1] = R::kBack ? mul(y[1], x[0][kb], d[1]) : mul(y[0], x[1][kb], d[1]);
        d[2] = mul(y[1], x[1][kb], d[2]);
      }
      f32x4_t m[3];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        m[0][r] = d[0][r] * (pair_factor[0][r] * x_factor[0]) * decays.pair[0][r];
        m[1][r] = d[1][r] * (pair_factor[R::kBack ? 1 : 0][r] * x_factor[R::kBack ? 0 : 1]) * decays.pair[1][r];
        m[2][r] = d[2][r] * (pair_factor[1][r] * x_factor[1]) * decays.pair[2][r];
        if constexpr (ROLE == kDecays) {
          m[0][r] *= decays.apart(0, 0, r);
          m[1][r] *= decays.apart(1, 0, r);
          m[2][r] *= decays.apart(1, 1, r);
        }
      }
      const f32x4_t none = {0, 0, 0, 0};
      const Pieces<3> sums[2] = {R::kBack ? cut<E::kPieces>(m[0], m[1]) : cut<E::kPieces>(m[0], none),
                                 R::kBack ? cut<E::kPieces>(none, m[2]) : cut<E::kPieces>(m[1], m[2])};
      // rows: 16 columns of this wave's (4g + r) of tokens 16 t + lane%16
      f32x4_t o[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      S.template cut_all<E::kPieces>();
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) {
        const Pieces<E::kPieces> both[2] = {x[0][kb], x[1][kb]};
        mul_right(S.p[kb], both, o);
      }
      if constexpr (ROLE == kDecays) {
        f32x4_t u[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
        T.template cut_all<E::kPieces>();
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
          const Pieces<E::kPieces> both[2] = {x[0][kb], x[1][kb]};
          mul_right(T.p[kb], both, u);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) o[t] = o[t] * decays.column[t] + u[t];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) o[t] *= x_factor[t] * decays.to[t];
      mul_right(z, sums, o);
      if constexpr (ROLE == kOut || ROLE == kDv) {
        const __amdgpu_buffer_rsrc_t r = s.of(ROLE == kOut ? a.O : a.dV, c, a.stride_row);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (ROLE == kDv && !((now >> (16 * t + (lane & 15))) & 1u)) o[t] = f32x4_t{0, 0, 0, 0};
          E::store_four(r, own_off + 16 * t * a.stride_row, o[t]);
        }
      } else if constexpr (ROLE == kDecays) {
        float of_chunk = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) of_chunk = ((now_there >> (16 * t + (lane & 15))) & 1u) ? fmaf(own.x[t][i], o[t][i], of_chunk) : of_chunk;
        sum += static_cast<double>(of_chunk);
      } else {
        held_live = R::kBack ? now : ~0u;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          held[t] = o[t];
          float dot = 0.0f, square = 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dot = fmaf(own.x[t][i], o[t][i], dot);
            square = fmaf(own.x[t][i], own.x[t][i], square);
          }
          dot = over_groups(dot);
          square = over_groups(square);
          if (group == 0) {
            parts[(wave * kChunk + 16 * t + lane) * 2] = dot;
            parts[(wave * kChunk + 16 * t + lane) * 2 + 1] = square;
          }
        }
      }
    }

    // the state: S <- a^n S + Y^T (w Z)
    count += decays.n;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v = 0.0f;
#pragma unroll
      for (int p = E::kPieces - 1; p >= 0; --p) v += static_cast<float>(z.p[p][i]);
      w[i] = v * (pair_factor[i >> 2][i & 3] * decays.fro[i >> 2][i & 3]);
    }
    if constexpr (R::kDerivative) {
      float wt[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) wt[i] = w[i] * (decays.n - decays.row[i >> 2][i & 3]);
      const Pieces<3> wz = cut<E::kPieces>(wt);
#pragma unroll
      for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = fmaf(decays.n, S.s[dt][i], T.s[dt][i]);
          T.s[dt][i] = fmaf(x, decays.whole_hi, x * decays.whole_lo);
        }
        T.s[dt] = mul(L::column_operand(smem + P::kY, dt, lane), wz, T.s[dt]);
      }
    }
#pragma unroll
    for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) S.s[dt][i] = fmaf(S.s[dt][i], decays.whole_hi, S.s[dt][i] * decays.whole_lo);
    delta::add_outer<L, D>(S, smem + P::kY, cut<E::kPieces>(w), lane);
    lds_barrier();
    if constexpr (R::kThrough) finish(c);
    if (c == last) break;
  }

  // what is behind the walk
  if constexpr (!R::kRows) {
    float* to = (R::kBack ? a.local_d : a.local_s) + (of_slice + segment) * D * D;
    S.store(to, col, lane);
    if constexpr (R::kDerivative) T.store(a.local_t + (of_slice + segment) * D * D, col, lane);
    if (threadIdx.x == 0) a.counts[of_slice + segment] = count;
  } else if constexpr (ROLE == kOut) {
    if (a.final_state != nullptr && segment == a.segments - 1) S.store(a.final_state + state_at, col, lane);
  } else if constexpr (ROLE == kDv) {
    if (a.dinitial_state != nullptr && segment == 0) S.store(a.dinitial_state + state_at, col, lane);
  } else if constexpr (ROLE == kDecays) {
    if (a.dfinal_state != nullptr && segment == a.segments - 1) {
      StateColumns<D> dS;
      dS.load(a.dfinal_state + state_at, col, lane);
#pragma unroll
      for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += static_cast<double>(dS.s[dt][i]) * static_cast<double>(T.s[dt][i]);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) a.dg[(of_slice + segment) * kWaves<D> + wave] = sum;
  }
}

}  // namespace decay
}  // namespace cotten
