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
  // of the state before it, and after a pass over them the state (derivative) before, and the gradient behind, each.
  float* local_s;               // [slice][segment][D][D]; at first the last one's place holds a copy of the initial state
  float* local_t;
  float* local_d;
  float* counts;                // [slice][segment][2]: how many of a segment's tokens count, and what they decay a state by
  double* dg;                   // [slice][segment][part]: partial sums of the decays' gradient
  int segments, segment_chunks;
  int unscanned;                // a forward's segments find the states before them from all local ones
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

// Powers of a head's decay, in LDS: a^n for n = 0 ... 32, and what rounding took from them.
struct Powers {
  float hi[kChunk + 4], lo[kChunk + 4];
};
// g * log2(e); a decay to nothing (g = -inf) counts as 2^-100000: fp32 knows no difference, and no tokens are none
__device__ __forceinline__ double rate_of(float g) {
  const double x = static_cast<double>(g) * 1.4426950408889634;
  return x < -100000.0 ? -100000.0 : x;
}
__device__ __forceinline__ void set_powers(Powers* to, double rate, int lane) {
  const double w = exp2(rate * static_cast<double>(lane));
  const float hi = static_cast<float>(w);
  if (lane <= kChunk) {
    to->hi[lane] = hi;
    to->lo[lane] = hi - hi == 0.0f ? static_cast<float>(w - static_cast<double>(hi)) : 0.0f;
  }
}

// p of a token of a chunk
__device__ __forceinline__ int upto(uint32_t live, int t) { return __popc(live & (0xffffffffu >> (31 - t))); }

// Two pieces of eight significant bits each, rounded: 16 bits, where a result of 11 or fewer is all that comes of them.
__device__ __forceinline__ Pieces<2> cut_in_two(const float (&x)[8]) {
  delta::u32x4_t h, m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    delta::bf16x2_t v;
    v[0] = static_cast<__bf16>(x[2 * i]);
    v[1] = static_cast<__bf16>(x[2 * i + 1]);
    uint32_t w = __builtin_bit_cast(uint32_t, v);
    asm("" : "+v"(w));  // (both halves from the one conversion)
    h[i] = w;
    v[0] = static_cast<__bf16>(x[2 * i] - __uint_as_float(w << 16));
    v[1] = static_cast<__bf16>(x[2 * i + 1] - delta::upper(__uint_as_float(w)));
    m[i] = __builtin_bit_cast(uint32_t, v);
  }
  Pieces<2> r;
  r.p[0] = __builtin_bit_cast(delta::bf16x8_t, h);
  r.p[1] = __builtin_bit_cast(delta::bf16x8_t, m);
  return r;
}
// What the rows of a result are made of: three pieces for fp32 results, two for 16-bit ones (a product is off by 2^-17, and a result
// rounded to 2^-9 or 2^-12 of it).
template <class E, int ROLE>
constexpr int kOperand = E::kBytes == 4 || ROLE == kDecays ? 3 : 2;
template <class E, int P>
__device__ __forceinline__ Pieces<P> cut_operand(f32x4_t a, f32x4_t b) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  if constexpr (P == 3) return cut<E::kPieces>(x);
  else return cut_in_two(x);
}

// The pairs of 16-token tiles that give each other anything: tile `x` of X's rows with tile `y` of Y's.  A wave makes every
// WAVES-th of the three.
template <class R>
struct Pair {
  int x, y;
  __device__ __forceinline__ explicit Pair(int i) : x(R::kBack ? i >> 1 : (i + 1) >> 1), y(R::kBack ? (i + 1) >> 1 : i >> 1) {}
};
// How many tokens of a chunk count, and the factors of a wave's pairs: columns lane%16 of X's tile, rows 4g + r of Y's.  Where all tokens
// from the first that counts to the last that exists count, pairs are as far apart as their numbers say, and the factors of the pairs are
// the same in all chunks.
template <class R, int WAVES, int COUNT = 3>
struct Decays {
  static constexpr int kOwn = (COUNT + WAVES - 1) / WAVES;           // pairs of a wave, at most (COUNT: 3 or, of two kinds of them, 6)
  uint32_t live;
  bool together;
  bool finite;              // all powers of a chunk
  float n;                  // tokens that count
  float pair[kOwn][4];
  float whole_hi, whole_lo;
  // tokens that count between column 16 x + lane%16 and row 16 y + 4g + r
  static __device__ __forceinline__ int apart(uint32_t live, const Pair<R>& p, int r, int lane) {
    const int column = upto(live, 16 * p.x + (lane & 15)), row = upto(live, 16 * p.y + 4 * (lane >> 4) + r);
    return R::kBack ? row - column : column - row;
  }
  __device__ __forceinline__ void set_pairs(uint32_t bits, const Powers* powers, int wave, int lane) {
    if constexpr (R::kRows) {
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int i = wave + k * WAVES;
        if (i >= COUNT) break;
        const Pair<R> p(i % 3);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 4 * (lane >> 4) + r, a = apart(bits, p, r, lane);
          const bool in = p.x != p.y || (R::kBack ? row >= (lane & 15) : row <= (lane & 15));
          const float w = powers->hi[a < 0 ? 0 : a];
          pair[k][r] = in ? w : 0.0f;
        }
      }
    }
  }
  __device__ __forceinline__ void begin(const Powers* powers, int wave, int lane) {
    none();
    together = true;
    finite = powers->hi[kChunk - 1] < __builtin_inff();
    set_pairs(~0u, powers, wave, lane);
  }
  // no token counts
  __device__ __forceinline__ void none() {
    live = 0;
    n = 0.0f;
    whole_hi = 1.0f;
    whole_lo = 0.0f;
  }
  // bits: at least one; `there`: the tokens that exist
  __device__ __forceinline__ void set(uint32_t bits, uint32_t there, const Powers* powers, int wave, int lane) {
    live = bits;
    const int count = __popc(bits);
    n = static_cast<float>(count);
    whole_hi = powers->hi[count];
    whole_lo = powers->lo[count];
    // (where the state grows, powers between tokens that do not count may be infinite, and are no factors of zeros)
    const bool now = finite && ((bits | ~there) >> __builtin_ctz(bits)) == (0xffffffffu >> __builtin_ctz(bits));
    if (!now || !together) set_pairs(now ? ~0u : bits, powers, wave, lane);
    together = now;
  }
};

// The first chunk of begin ... end-1 with a token that counts, or `end`.
__device__ __forceinline__ int first_live(const uint8_t* mask, int N, int begin, int end, int lane) {
  const __amdgpu_buffer_rsrc_t r = buffer(mask, N);
  for (int t = kChunk * begin; t < N && t < kChunk * end; t += 256) {
    uint8_t b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) b[u] = __builtin_amdgcn_raw_buffer_load_b8(r, static_cast<uint32_t>(t + 64 * u + lane), 0, 0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint64_t votes = __ballot(b[u] != 0);
      if (votes != 0) {
        const int c = (t + 64 * u + static_cast<int>(__builtin_ctzll(votes))) / kChunk;
        return c < end ? c : end;
      }
    }
  }
  return end;
}

// Whether no token of the first `chunks` counts: 1024 of them at a time (more would take registers that the states are in).
__device__ __forceinline__ bool none_before(const uint8_t* mask, int chunks, int lane) {
  typedef delta::u32x4_t __attribute__((aligned(1))) bytes;  // (rows of a mask begin anywhere)
  const bytes* of = reinterpret_cast<const bytes*>(mask);
#pragma unroll 1
  for (int at = 0; at < 2 * chunks; at += 64) {  // (the same in all lanes)
    delta::u32x4_t x = {0, 0, 0, 0};
    if (at + lane < 2 * chunks) x = of[at + lane];
    if (__ballot((x[0] | x[1] | x[2] | x[3]) != 0) != 0) return false;
  }
  return true;
}

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

// A chunk's place in LDS: rows in pieces; by token the factors of X's rows and of Y's and Z's, and both with what decays between them and
// the state.
template <class E, int D, bool ROWS>
struct Place {
  typedef Rows<D, E::kPieces> R;
  static constexpr int kY = 0, kZ = R::kBytes, kX = 2 * R::kBytes, kOfX = ROWS ? 3 * R::kBytes : 2 * R::kBytes;
  static constexpr int kOfPair = kOfX + kChunk * 4, kTo = kOfPair + kChunk * 4, kOfState = kTo + kChunk * 4, kPowers = kOfState + kChunk * 4, kBytes = kPowers + static_cast<int>(sizeof(Powers));
};
// ... followed by the products of the pairs of tiles as operands ([tile of X][piece][lane], 16 bytes), and what waves sum over all columns.
template <int OF>
constexpr int kPairBytes = 2 * OF * 64 * 16;
template <class E, int D, int ROLE>
constexpr int kLds = Place<E, D, Traits<ROLE>::kRows>::kBytes + (Traits<ROLE>::kRows ? kPairBytes<kOperand<E, ROLE>> : 0) +
                     (Traits<ROLE>::kThrough ? kWaves<D> * kChunk * 8 : 0);
// Four values of a lane as half of an operand.
template <class E, int OF>
__device__ __forceinline__ void put_half(unsigned char* at, int tile, int half, int lane, f32x4_t x) {
  const Pieces<OF> p = cut_operand<E, OF>(x, f32x4_t{0, 0, 0, 0});
#pragma unroll
  for (int i = 0; i < OF; ++i) {
    const delta::u32x4_t w = __builtin_bit_cast(delta::u32x4_t, p.p[i]);
    *reinterpret_cast<delta::u32x2_t*>(at + ((tile * OF + i) * 64 + lane) * 16 + 8 * half) = delta::u32x2_t{w[0], w[1]};
  }
}
template <int OF>
__device__ __forceinline__ Pieces<OF> pair_operand(const unsigned char* at, int tile, int lane) {
  Pieces<OF> r;
#pragma unroll
  for (int i = 0; i < OF; ++i) r.p[i] = *reinterpret_cast<const delta::bf16x8_t*>(at + ((tile * OF + i) * 64 + lane) * 16);
  return r;
}

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
  float s = 0.0f;
  if constexpr (E::kBytes == 2 && E::kPieces == 1) {  // bf16: pairs as they are, 4 instructions for 16
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = raw[i];  // (a bit cast of an element in place takes the first)
      const pair x = __builtin_bit_cast(pair, w);
      s = __builtin_amdgcn_fdot2_f32_bf16(x, x, s, false);
    }
  } else {
    float x[8];
    E::unpack(raw, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
  }
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

// The walk of one unit: a slice, or a segment of it.  Every wave carries 16 columns of the state; all load the chunk's rows (eight
// elements a lane) and leave them in LDS in pieces.  GROUPS: workgroups that share the columns of a unit, each with all rows.
template <class E, int D, int ROLE, int GROUPS = 1>
__device__ void walk(const Args& a, int unit, unsigned char* smem, int part = 0) {
  static_assert(GROUPS == 1 || !Traits<ROLE>::kThrough, "sums over all columns are a workgroup's");
  constexpr int kWavesHere = kWaves<D> / GROUPS, kRowsOfPass = kWavesHere * (512 / D);
  typedef Traits<ROLE> R;
  typedef Place<E, D, R::kRows> P;
  typedef typename P::R L;
  constexpr int kOf = kOperand<E, ROLE>, kRowLanes = D / 8, kBlocks = StateColumns<D>::kBlocks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slice = unit / a.segments, segment = unit - slice * a.segments;
  const Slice s(a, slice, D * E::kBytes);
  const double rate = rate_of(s.g);
  int begin = segment * a.segment_chunks;
  const int end = begin + a.segment_chunks < a.chunks ? begin + a.segment_chunks : a.chunks;
  const int tile = part * kWavesHere + wave, col = 16 * tile + (lane & 15), group = lane >> 4;
  const long long of_slice = static_cast<long long>(slice) * a.segments;
  const long long state_at = static_cast<long long>(slice) * D * D;
  float* of_x = reinterpret_cast<float*>(smem + P::kOfX);
  float* of_pair = reinterpret_cast<float*>(smem + P::kOfPair);
  float* to_state = reinterpret_cast<float*>(smem + P::kTo);
  float* of_state = reinterpret_cast<float*>(smem + P::kOfState);

  Powers* powers = reinterpret_cast<Powers*>(smem + P::kPowers);
  unsigned char* pairs = smem + P::kBytes;
  if (D < 32)  // narrow rows are followed by zeros
    for (int i = threadIdx.x; i < P::kOfX / 16; i += 64 * kWavesHere) reinterpret_cast<f32x4_t*>(smem)[i] = f32x4_t{0, 0, 0, 0};
  if (R::kRows)  // so are the pairs that give each other nothing
    for (int i = threadIdx.x; i < kPairBytes<kOf> / 16; i += 64 * kWavesHere) reinterpret_cast<f32x4_t*>(pairs)[i] = f32x4_t{0, 0, 0, 0};
  if (wave == 0) set_powers(powers, rate, lane);
  lds_barrier();

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
  } else if (a.segments == 1 || (R::kBack && segment == a.segments - 1)) {
    load_state<D, R::kTransposed>(S, outer, col, lane);
  } else if (ROLE == kOut && a.unscanned) {
    // what the segments before add, the first's with the initial state in it
    const float* local = a.local_s + of_slice * D * D;
    S.load(local + static_cast<long long>(segment == 0 ? a.segments - 1 : 0) * D * D, col, lane);
    constexpr int kAhead = D == 128 ? 2 : 4;  // on their way together
    for (int i = 1; i < segment; i += kAhead) {
      StateColumns<D> x[kAhead];
      float w[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        x[u].load(i + u < segment ? local + static_cast<long long>(i + u) * D * D : nullptr, col, lane);
        w[u] = i + u < segment ? a.counts[2 * (of_slice + i + u) + 1] : 1.0f;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int dt = 0; dt < 2 * kBlocks; ++dt) S.s[dt] = S.s[dt] * w[u] + x[u].s[dt];
    }
  } else {
    load_state<D, R::kTransposed>(S, (R::kBack ? a.local_d : a.local_s) + (of_slice + segment) * D * D, col, lane);
    if constexpr (R::kDerivative) load_state<D, false>(T, a.local_t + (of_slice + segment) * D * D, col, lane);
  }

  // Chunks at a unit's beginning without a token that counts, skipped: forwards where no state comes from outside, back where nobody
  // asks for the gradient of one.  They add nothing to a forward's local states, and keys and values have no gradients there.  Rows of O and dQ (and
  // their share of dg) are zeros at once only where no token before the unit counts either, as queries read the state that those left; and what
  // queries add to dS is nobody's only where there is no key before them.  That is looked up where it can save more chunks (1.2 us each)
  // than it takes rounds (0.6).
  const int row = wave * (512 / D) + lane / kRowLanes;
  const uint32_t off = static_cast<uint32_t>(row) * a.stride_row + (lane % kRowLanes) * 8 * E::kBytes;
  if (a.mask != nullptr && (R::kBack ? (ROLE == kDk || a.dinitial_state == nullptr) : a.initial_state == nullptr)) {
    int from = first_live(s.mask, a.N, begin, end, lane);
    if constexpr (ROLE == kOut || ROLE == kDq || ROLE == kDecays || ROLE == kGradStates)
      if (from > begin && begin > 0 && (begin > 32 * (from - begin) || !none_before(s.mask, begin, lane))) from = begin;
    if constexpr (R::kRows && ROLE != kDecays) {
      unsigned char* to = ROLE == kOut ? a.O : ROLE == kDq ? a.dQ : ROLE == kDk ? a.dK : a.dV;
      for (int c = begin; c < from; ++c) {
        const __amdgpu_buffer_rsrc_t r = s.of(to, c, a.stride_row);
        // (of the columns' groups, each its share of the rows)
        E::store_four(r, off + part * kRowsOfPass * a.stride_row, f32x4_t{0, 0, 0, 0});
        E::store_four(r, off + part * kRowsOfPass * a.stride_row + 4 * E::kBytes, f32x4_t{0, 0, 0, 0});
      }
    }
    begin = from;
  }

  Mask mask(a, s);
  uint32_t live = 0, there = 0;
  typename E::Raw rx[GROUPS], ry[GROUPS], rz[GROUPS];   // by passes over the chunk's rows
  ResultRows<E> own;                        // rows of Q or K (through their norm), or of dO (decays)
  const uint32_t own_off = static_cast<uint32_t>(lane & 15) * a.stride_row + (16 * tile + 4 * group) * E::kBytes;
  auto fetch = [&](int chunk) {
    live = mask.bits(chunk);
    there = existing(a.N, chunk);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      // forwards the mask is that of Y and Z, back that of X
      const uint32_t here = off + i * kRowsOfPass * a.stride_row, masked = offset_if(live, row + i * kRowsOfPass, here);
      const uint32_t at_x = R::kBack ? masked : here, at_yz = R::kBack ? here : masked;
      if constexpr (R::kRows) rx[i] = E::load(s.of(R::x(a), chunk, a.stride_row), at_x);
      ry[i] = E::load(s.of(R::y(a), chunk, a.stride_row), at_yz);
      rz[i] = E::load(s.of(R::z(a), chunk, a.stride_row), at_yz);
    }
  };
  const int step = R::kBack ? -1 : 1, first = R::kBack ? end - 1 : begin, last = R::kBack ? begin : end - 1;
  const int walked = end - begin;           // (may be none)
  if (walked > 0) {
    mask.fetch(first, lane);
    fetch(first);
    if (first != last) mask.fetch(first + step, lane);
  }
  Decays<R, kWavesHere> decays;
  decays.begin(powers, wave, lane);
  float count = 0.0f;
  double sum = 0.0;
  f32x4_t held[2];                          // rows that wait for the sums over the waves
  uint32_t held_live = 0;
  float* parts = reinterpret_cast<float*>(pairs + kPairBytes<kOf>);   // [wave][token]: y . x^ and y . y
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

  for (int i = 0, c = first; i < walked; ++i, c += step) {
    // rows to LDS
    const uint32_t now = live, now_there = there;
    // where no token counts, forwards nothing is added to the state, and back there are no rows
    const bool dead = now == 0, with_rows = !R::kBack || !dead, with_sums = R::kBack || !dead;
#pragma unroll
    for (int n = 0; n < GROUPS; ++n) {
      const int kb = (lane % kRowLanes) / 4, g = (lane % kRowLanes) % 4, of = row + n * kRowsOfPass;
      float fx = 1.0f, fyz = 1.0f;
      if constexpr (R::kRows) {
        if (with_rows) {
          L::put(smem + P::kX, of, kb, g, E::pieces(rx[n]));
          if constexpr (R::kUnitX) fx = inverse_norm<E, D>(rx[n], a.eps);
        }
      }
      if (with_sums) {
        L::put(smem + P::kY, of, kb, g, E::pieces(ry[n]));
        L::put(smem + P::kZ, of, kb, g, E::pieces(rz[n]));
        fyz = inverse_norm<E, D>(R::kUnitY ? ry[n] : rz[n], a.eps);
      }
      if (R::kScaleX) fx *= a.scale;
      else fyz *= a.scale;
      const uint32_t in_x = R::kBack ? now : now_there, in_yz = R::kBack ? now_there : now;
      const int p = upto(now, of), behind = __popc(now) - p;
      fyz = ((in_yz >> of) & 1u) ? fyz : 0.0f;
      if (lane % kRowLanes == 0) {
        if (R::kRows) {
          of_x[of] = ((in_x >> of) & 1u) ? fx : 0.0f;
          to_state[of] = powers->hi[R::kBack ? behind : p];
        }
        of_pair[of] = fyz;
        of_state[of] = fyz * powers->hi[R::kBack ? p : behind];
      }
    }
    if (now != decays.live) {
      if (dead) decays.none();
      else decays.set(now, now_there, powers, wave, lane);
    }
    if (c != last) {
      fetch(c + step);
      if (c + step != last) mask.fetch(c + 2 * step, lane);
    }
    lds_barrier();

    if constexpr (R::kThrough)
      if (i > 0) finish(c - step);
    Pieces<E::kPieces> z;
    if (with_sums) z = L::column_operand(smem + P::kZ, tile, lane);
    // rows: 16 columns of this wave's (4g + r) of tokens 16 t + lane%16
    f32x4_t o[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    float x_factor[2] = {0.0f, 0.0f};
    if constexpr (R::kRows) {
      if constexpr (R::kThrough || ROLE == kDecays)
        own.load(s.of(ROLE == kDq ? a.Q : ROLE == kDk ? a.K : a.dO, c, a.stride_row), a.stride_row, R::kBack ? now : ~0u, own_off, lane);
      // this wave's share of the products of X's rows with Y's (rows Y, columns X), for all
      if (!dead) {
#pragma unroll
        for (int k = 0; k < decays.kOwn; ++k) {
          const int p = wave + k * kWavesHere;
          if (p >= 3) break;
          const Pair<R> pair(p);
          f32x4_t m = {0, 0, 0, 0};
#pragma unroll
          for (int kb = 0; kb < kBlocks; ++kb)
            m = mul(L::row_operand(smem + P::kY, pair.y, kb, lane), L::row_operand(smem + P::kX, pair.x, kb, lane), m);
          const f32x4_t factor = *reinterpret_cast<const f32x4_t*>(of_pair + 16 * pair.y + 4 * group);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            m[r] *= factor[r] * decays.pair[k][r];
            if constexpr (ROLE == kDecays) m[r] *= static_cast<float>(decays.apart(now, pair, r, lane));
          }
          put_half<E, kOf>(pairs, pair.x, pair.y, lane, m);
        }
      }
      if (with_rows) {
        x_factor[0] = of_x[lane & 15];
        x_factor[1] = of_x[16 + (lane & 15)];
        f32x4_t u[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
          const Pieces<E::kPieces> both[2] = {L::row_operand(smem + P::kX, 0, kb, lane), L::row_operand(smem + P::kX, 1, kb, lane)};
          mul_right(cut_operand<E, kOf>(S.s[2 * kb], S.s[2 * kb + 1]), both, o);
          if constexpr (ROLE == kDecays) mul_right(cut_operand<E, kOf>(T.s[2 * kb], T.s[2 * kb + 1]), both, u);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (ROLE == kDecays) o[t] = o[t] * static_cast<float>(upto(now, 16 * t + (lane & 15))) + u[t];
          o[t] *= to_state[16 * t + (lane & 15)];
        }
      }
    }

    // the state: S <- a^n S + Y^T (w Z)
    if (with_sums) {
      count += decays.n;
      const f32x4_t factor[2] = {*reinterpret_cast<const f32x4_t*>(of_state + 4 * group), *reinterpret_cast<const f32x4_t*>(of_state + 16 + 4 * group)};
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = 0.0f;
#pragma unroll
        for (int p = E::kPieces - 1; p >= 0; --p) v += static_cast<float>(z.p[p][j]);
        w[j] = v * factor[j >> 2][j & 3];
      }
      if constexpr (R::kDerivative) {
        float wt[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) wt[j] = w[j] * (decays.n - static_cast<float>(upto(now, 16 * (j >> 2) + 4 * group + (j & 3))));
        const Pieces<3> wz = cut<E::kPieces>(wt);
#pragma unroll
        for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = fmaf(decays.n, S.s[dt][j], T.s[dt][j]);
            T.s[dt][j] = fmaf(x, decays.whole_hi, x * decays.whole_lo);
          }
          T.s[dt] = mul(L::column_operand(smem + P::kY, dt, lane), wz, T.s[dt]);
        }
      }
#pragma unroll
      for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) S.s[dt][j] = fmaf(S.s[dt][j], decays.whole_hi, S.s[dt][j] * decays.whole_lo);
      delta::add_outer<L, D>(S, smem + P::kY, cut<E::kPieces>(w), lane);
    }
    lds_barrier();

    // what the chunk's tokens give each other; the next chunk's rows may be written from here on
    if constexpr (R::kRows) {
      if (!dead) {
        const Pieces<kOf> sums[2] = {pair_operand<kOf>(pairs, 0, lane), pair_operand<kOf>(pairs, 1, lane)};
        mul_right(z, sums, o);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) o[t] *= x_factor[t];
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
          for (int j = 0; j < 4; ++j) of_chunk = ((now_there >> (16 * t + (lane & 15))) & 1u) ? fmaf(own.x[t][j], o[t][j], of_chunk) : of_chunk;
        sum += static_cast<double>(of_chunk);
      } else {
        held_live = R::kBack ? now : ~0u;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          held[t] = o[t];
          float dot = 0.0f, square = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            dot = fmaf(own.x[t][j], o[t][j], dot);
            square = fmaf(own.x[t][j], own.x[t][j], square);
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
  }
  if constexpr (R::kThrough) {
    lds_barrier();
    if (walked > 0) finish(first + (walked - 1) * step);
  }

  // what is behind the walk
  if constexpr (!R::kRows) {
    float* to = (R::kBack ? a.local_d : a.local_s) + (of_slice + segment) * D * D;
    S.store(to, col, lane);
    if constexpr (R::kDerivative) T.store(a.local_t + (of_slice + segment) * D * D, col, lane);
    if (threadIdx.x == 0) {
      a.counts[2 * (of_slice + segment)] = count;
      a.counts[2 * (of_slice + segment) + 1] = static_cast<float>(exp2(rate * static_cast<double>(count)));
    }
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
    if (lane == 0) a.dg[(of_slice + segment) * kWaves<D> + tile] = sum;
  }
}

// The gradients of keys and values in one walk, for wide 16-bit rows: both go back with dS, by columns in the waves, so its update and the rows
// of Q and dO are shared.  dV takes a wave's own columns of dS, dK those of dS^T, which all waves leave in LDS in pieces, behind the second
// barrier of a chunk, for the next.  A chunk takes half as long again as one of either gradient by itself.
template <class E, int D>
struct BackPlace {
  static_assert(D >= 32 && E::kBytes == 2, "rows without zeros behind them, results of two pieces");
  static constexpr int kOf = kOperand<E, kDv>;
  typedef Rows<D, E::kPieces> R;
  typedef Rows<D, kOf> M;                      // 32 columns of dS a block
  static constexpr int kBlocks = StateColumns<D>::kBlocks;
  static constexpr int kQ = 0, kO = R::kBytes, kK = 2 * R::kBytes, kV = 3 * R::kBytes, kState = 4 * R::kBytes, kOfK = kState + kBlocks * M::kBytes;
  static constexpr int kOfPair = kOfK + kChunk * 4, kTo = kOfPair + kChunk * 4, kOfState = kTo + kChunk * 4, kPowers = kOfState + kChunk * 4;
  static constexpr int kPairs = kPowers + static_cast<int>(sizeof(Powers)), kParts = kPairs + 2 * kPairBytes<kOf>;
  static constexpr int kBytes = kParts + kWaves<D> * kChunk * 8;
};
template <class E, int D>
__device__ void walk_back(const Args& a, int unit, unsigned char* smem) {
  typedef Traits<kDv> T;
  typedef BackPlace<E, D> P;
  typedef typename P::R L;
  typedef typename P::M M;
  constexpr int kOf = P::kOf, kRowLanes = D / 8, kBlocks = P::kBlocks, kW = kWaves<D>, kEach = kPairBytes<kOf>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slice = unit / a.segments, segment = unit - slice * a.segments;
  const Slice s(a, slice, D * E::kBytes);
  int begin = segment * a.segment_chunks;
  const int end = begin + a.segment_chunks < a.chunks ? begin + a.segment_chunks : a.chunks;
  const int col = 16 * wave + (lane & 15), group = lane >> 4;
  const long long of_slice = static_cast<long long>(slice) * a.segments, state_at = static_cast<long long>(slice) * D * D;
  float* of_k = reinterpret_cast<float*>(smem + P::kOfK);
  float* of_pair = reinterpret_cast<float*>(smem + P::kOfPair);
  float* to_state = reinterpret_cast<float*>(smem + P::kTo);
  float* of_state = reinterpret_cast<float*>(smem + P::kOfState);
  float* parts = reinterpret_cast<float*>(smem + P::kParts);       // [wave][token]: k . dk^ and k . k
  Powers* powers = reinterpret_cast<Powers*>(smem + P::kPowers);
  unsigned char* pairs = smem + P::kPairs;                         // of dV, and behind them of dK
  for (int i = threadIdx.x; i < 2 * kEach / 16; i += 64 * kW) reinterpret_cast<f32x4_t*>(pairs)[i] = f32x4_t{0, 0, 0, 0};
  if (wave == 0) set_powers(powers, rate_of(s.g), lane);
  lds_barrier();

  StateColumns<D> S;
  const bool outermost = a.segments == 1 || segment == a.segments - 1;
  S.load(!outermost ? a.local_d + (of_slice + segment) * D * D : a.dfinal_state == nullptr ? nullptr : a.dfinal_state + state_at, col, lane);
  auto hand_over = [&]() {
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      const Pieces<kOf> x = cut_operand<E, kOf>(S.s[2 * kb], S.s[2 * kb + 1]);
      unsigned char* to = smem + P::kState + (col >> 5) * M::kBytes + (col & 31) * M::kStride + kb * 64 + 16 * group;
#pragma unroll
      for (int i = 0; i < kOf; ++i) *reinterpret_cast<delta::bf16x8_t*>(to + i * M::kPlane) = x.p[i];
    }
  };

  const int row = wave * (512 / D) + lane / kRowLanes;
  const uint32_t off = static_cast<uint32_t>(row) * a.stride_row + (lane % kRowLanes) * 8 * E::kBytes;
  if (a.mask != nullptr && a.dinitial_state == nullptr) {  // chunks before the first token that counts
    const int from = first_live(s.mask, a.N, begin, end, lane);
    for (int c = begin; c < from; ++c) {
      const __amdgpu_buffer_rsrc_t rk = s.of(a.dK, c, a.stride_row), rv = s.of(a.dV, c, a.stride_row);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        E::store_four(rk, off + 4 * i * E::kBytes, f32x4_t{0, 0, 0, 0});
        E::store_four(rv, off + 4 * i * E::kBytes, f32x4_t{0, 0, 0, 0});
      }
    }
    begin = from;
  }

  Mask mask(a, s);
  uint32_t live = 0, there = 0;
  typename E::Raw rq, ro, rk, rv;
  ResultRows<E> own;                        // rows of K
  const uint32_t own_off = static_cast<uint32_t>(lane & 15) * a.stride_row + (16 * wave + 4 * group) * E::kBytes;
  auto fetch = [&](int chunk) {
    live = mask.bits(chunk);
    there = existing(a.N, chunk);
    const uint32_t masked = offset_if(live, row, off);
    rq = E::load(s.of(a.Q, chunk, a.stride_row), off);
    ro = E::load(s.of(a.dO, chunk, a.stride_row), off);
    rk = E::load(s.of(a.K, chunk, a.stride_row), masked);
    rv = E::load(s.of(a.V, chunk, a.stride_row), masked);
  };
  const int first = end - 1, last = begin;
  if (end > begin) {
    mask.fetch(first, lane);
    fetch(first);
    if (first != last) mask.fetch(first - 1, lane);
    hand_over();
  }
  Decays<T, kW, 6> decays;
  decays.begin(powers, wave, lane);
  f32x4_t held[2];                          // rows of dk^ that wait for the sums over the waves
  uint32_t held_live = 0;
  auto finish = [&](int chunk) {
    const __amdgpu_buffer_rsrc_t r = s.of(a.dK, chunk, a.stride_row);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int token = 16 * t + (lane & 15);
      float dot = 0.0f, square = 0.0f;
#pragma unroll
      for (int w = 0; w < kW; ++w) {
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

  for (int c = first; c >= last; --c) {
    const uint32_t now = live, now_there = there;
    const bool dead = now == 0;             // no rows of keys and values
    {
      const int kb = (lane % kRowLanes) / 4, g = (lane % kRowLanes) % 4;
      L::put(smem + P::kQ, row, kb, g, E::pieces(rq));
      L::put(smem + P::kO, row, kb, g, E::pieces(ro));
      float fk = 0.0f;
      if (!dead) {
        L::put(smem + P::kK, row, kb, g, E::pieces(rk));
        L::put(smem + P::kV, row, kb, g, E::pieces(rv));
        fk = inverse_norm<E, D>(rk, a.eps);
      }
      const float norm = a.scale * inverse_norm<E, D>(rq, a.eps), fq = ((now_there >> row) & 1u) ? norm : 0.0f;
      const int p = upto(now, row), behind = __popc(now) - p;
      if (lane % kRowLanes == 0) {
        of_k[row] = ((now >> row) & 1u) ? fk : 0.0f;
        to_state[row] = powers->hi[behind];
        of_pair[row] = fq;
        of_state[row] = fq * powers->hi[p];
      }
    }
    if (now != decays.live) {
      if (dead) decays.none();
      else decays.set(now, now_there, powers, wave, lane);
    }
    if (c != last) {
      fetch(c - 1);
      if (c - 1 != last) mask.fetch(c - 2, lane);
    }
    lds_barrier();

    if (c != first) finish(c + 1);
    f32x4_t of_v[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}}, of_keys[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    own.load(s.of(a.K, c, a.stride_row), a.stride_row, now, own_off, lane);
    const Pieces<E::kPieces> z = L::column_operand(smem + P::kO, wave, lane);
    if (!dead) {
      // this wave's share of the products of pairs, for all: q . k for dV, dO . v for dK
#pragma unroll
      for (int k = 0; k < decays.kOwn; ++k) {
        const int i = wave + k * kW;
        if (i >= 6) break;
        const Pair<T> pair(i % 3);
        const unsigned char* y = smem + (i < 3 ? P::kQ : P::kO);
        const unsigned char* x = smem + (i < 3 ? P::kK : P::kV);
        f32x4_t m = {0, 0, 0, 0};
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) m = mul(L::row_operand(y, pair.y, kb, lane), L::row_operand(x, pair.x, kb, lane), m);
        const f32x4_t factor = *reinterpret_cast<const f32x4_t*>(of_pair + 16 * pair.y + 4 * group);
#pragma unroll
        for (int r = 0; r < 4; ++r) m[r] *= factor[r] * decays.pair[k][r];
        put_half<E, kOf>(pairs + (i < 3 ? 0 : kEach), pair.x, pair.y, lane, m);
      }
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) {
        const unsigned char* mine = smem + P::kState + (col >> 5) * M::kBytes + (col & 31) * M::kStride + kb * 64 + 16 * group;
        Pieces<kOf> x;
#pragma unroll
        for (int i = 0; i < kOf; ++i) x.p[i] = *reinterpret_cast<const delta::bf16x8_t*>(mine + i * M::kPlane);
        const Pieces<E::kPieces> keys[2] = {L::row_operand(smem + P::kK, 0, kb, lane), L::row_operand(smem + P::kK, 1, kb, lane)};
        mul_right(x, keys, of_v);
        const Pieces<E::kPieces> values[2] = {L::row_operand(smem + P::kV, 0, kb, lane), L::row_operand(smem + P::kV, 1, kb, lane)};
        mul_right(M::column_operand(smem + P::kState + kb * M::kBytes, wave, lane), values, of_keys);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float w = to_state[16 * t + (lane & 15)];
        of_v[t] *= w;
        of_keys[t] *= w;
      }
    }

    // the state: dS <- a^n dS + Q^T (w dO)
    {
      const f32x4_t factor[2] = {*reinterpret_cast<const f32x4_t*>(of_state + 4 * group), *reinterpret_cast<const f32x4_t*>(of_state + 16 + 4 * group)};
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = 0.0f;
#pragma unroll
        for (int p = E::kPieces - 1; p >= 0; --p) v += static_cast<float>(z.p[p][j]);
        w[j] = v * factor[j >> 2][j & 3];
      }
#pragma unroll
      for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) S.s[dt][j] = fmaf(S.s[dt][j], decays.whole_hi, S.s[dt][j] * decays.whole_lo);
      delta::add_outer<L, D>(S, smem + P::kQ, cut<E::kPieces>(w), lane);
    }
    const float scale_k[2] = {of_k[lane & 15], of_k[16 + (lane & 15)]};
    Pieces<E::kPieces> y;
    if (!dead) y = L::column_operand(smem + P::kQ, wave, lane);
    lds_barrier();

    // what the chunk's tokens give each other; the next chunk's rows, and dS before this one, may be written from here on
    if (c != last) hand_over();
    if (!dead) {
      const Pieces<kOf> for_v[2] = {pair_operand<kOf>(pairs, 0, lane), pair_operand<kOf>(pairs, 1, lane)};
      mul_right(z, for_v, of_v);
      const Pieces<kOf> for_k[2] = {pair_operand<kOf>(pairs + kEach, 0, lane), pair_operand<kOf>(pairs + kEach, 1, lane)};
      mul_right(y, for_k, of_keys);
    }
    const __amdgpu_buffer_rsrc_t r = s.of(a.dV, c, a.stride_row);
    held_live = now;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      of_v[t] *= scale_k[t];
      if (!((now >> (16 * t + (lane & 15))) & 1u)) of_v[t] = f32x4_t{0, 0, 0, 0};
      E::store_four(r, own_off + 16 * t * a.stride_row, of_v[t]);
      held[t] = of_keys[t];
      float dot = 0.0f, square = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dot = fmaf(own.x[t][j], of_keys[t][j], dot);
        square = fmaf(own.x[t][j], own.x[t][j], square);
      }
      dot = over_groups(dot);
      square = over_groups(square);
      if (group == 0) {
        parts[(wave * kChunk + 16 * t + lane) * 2] = dot;
        parts[(wave * kChunk + 16 * t + lane) * 2 + 1] = square;
      }
    }
  }
  lds_barrier();
  if (end > begin) finish(last);
  if (a.dinitial_state != nullptr && segment == 0) S.store(a.dinitial_state + state_at, col, lane);
}

}  // namespace decay
}  // namespace cotten
