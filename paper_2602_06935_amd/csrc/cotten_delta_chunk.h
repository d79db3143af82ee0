// The waves of the chunked kernels of the gated delta rule (see cotten_delta_core.h for the formulas): two producers that
// make what a chunk needs besides the state, and consumers that carry 16 columns of the state each.
#pragma once
#include "cotten_delta_core.h"

namespace cotten {
namespace delta {

// The role of a wave in a workgroup of WAVES.  Four waves take one SIMD each, and the producers would sit on the same two in
// every workgroup of a compute unit: they move on by one from each 256 workgroups to the next (256 x 2 x 200 x 32 fp32,
// forward: 23.9 -> 21.2 us; workgroups of six waves are spread by the hardware, and lose by it).
template <int WAVES>
__device__ __forceinline__ int role_of_wave() {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  return WAVES == 4 ? (wave + 3 * (blockIdx.x >> 8)) % 4 : wave;
}

// One chunk's place in LDS.  The producers fill one while the consumers read the other.
template <class E, int D, bool QUERIES>
struct ChunkBuffer {
  typedef Rows<D, E::kPieces> R;
  static constexpr int kK = 0, kT = R::kBytes, kQ = kT + kTriangleBytes, kM = kQ + R::kBytes;
  static constexpr int kCoef = QUERIES ? kM + kTriangleBytes : kQ;
  static constexpr int kBytes = kCoef + (5 * kChunk + 4) * 4;
  // coefficients by token: four columns, and e^(G_C) behind them
  enum { kBeta = 0, kReadK = kChunk, kWriteK = 2 * kChunk, kQuery = 3 * kChunk, kAdjoint = 4 * kChunk, kWhole = 5 * kChunk };
};

// Waves on a SIMD that the registers of a walk must leave room for: those of two workgroups of WAVES on a compute unit, where
// their LDS leaves room for two (128 x 4 x 200 x 64 bf16: 26 us, and 32 where registers admitted one), but not more than three
// (168 registers; the nine waves of a transition would get 96, and spill).
constexpr int waves_per_simd(int waves, int lds) {
  const int of_two = (2 * waves + 3) / 4;
  return lds > 80 * 1024 ? (waves + 3) / 4 : of_two < 3 ? of_two : 3;
}

// Producer of the keys: rows of K in pieces, T (backward: T^T), and the coefficients
//     kReadK  r e^G (what K S is multiplied with)     kWriteK  r e^(G_C - G)     kAdjoint  -beta e^G r (backward)
template <class E, int D, bool BWD, bool QUERIES>
struct KeyProducer {
  typedef ChunkBuffer<E, D, QUERIES> B;
  const Args& a;
  const Live lives;
  const Slice& s;
  const __amdgpu_buffer_rsrc_t decays, betas;
  RowTile<E, D> k;
  uint32_t live, g, beta;  // (gates as they were loaded)
  uint32_t byte;

  __device__ __forceinline__ KeyProducer(const Args& args, const Slice& slice)
      : a(args), lives(args, slice), s(slice), decays(slice.of_gate(args, args.g)), betas(slice.of_gate(args, args.beta)) {}
  __device__ __forceinline__ void fetch(int chunk, int lane) {
    live = lives.bits(byte, chunk);
    k.load(s.of(a.K, chunk, a.stride_row), a.stride_row, live, lane);
    g = fetch_gate(a, decays, chunk, live, lane);
    beta = fetch_gate(a, betas, chunk, live, lane);
  }
  // the first chunk, and the mask of the next
  __device__ __forceinline__ void begin(int chunk, int next, int lane) {
    byte = lives.fetch(chunk, lane);
    fetch(chunk, lane);
    byte = lives.fetch(next, lane);
  }
  // makes the chunk that was fetched; begins the loads of `next` (negative or beyond the last: none), and of the mask of `after`
  __device__ __forceinline__ void make(int next, int after, unsigned char* at, Scratch* scratch, int lane) {
    const int c = lane & 15, gr = lane >> 4;
    float* coef = reinterpret_cast<float*>(at + B::kCoef);
    k.put(at + B::kK, lane);
    const Sum G = scan_decays(__uint_as_float(g), lane), G_end = last_of_scan(G);
    // k_i . k_j: backward keeps the lower block as its transpose, see below
    const f32x4_t d00 = dots(k, 0, k, 0), d11 = dots(k, 1, k, 1), d10 = BWD ? dots(k, 0, k, 1) : dots(k, 1, k, 0);
    const float rn0 = inverse_norm(d00, 0, a.eps, live, lane), rn1 = inverse_norm(d11, 1, a.eps, live, lane);
    if (lane < 32) {
      const float r = lane < 16 ? rn0 : rn1, eG = pow2(G), b = __uint_as_float(beta);
      scratch->notes.hi[lane] = G.hi;
      scratch->notes.lo[lane] = G.lo;
      scratch->notes.factor[lane] = b * r;
      if (BWD) scratch->notes.other[lane] = r;
      coef[B::kBeta + lane] = b;
      coef[B::kReadK + lane] = r * eG;
      coef[B::kWriteK + lane] = r * pow2(G_end, G);
      if (BWD) coef[B::kAdjoint + lane] = -b * eG * r;
      if (lane == 31) coef[B::kWhole] = eG;
    }
    // the next chunk's rows, while this one is worked on
    if (next >= 0 && next < a.chunks) {
      fetch(next, lane);
      byte = lives.fetch(after, lane);
    }
    wave_fence();
    const Noted n(scratch->notes, lane);
    f32x4_t a00, a11, a10;
    f32x4_t by_key = {0, 0, 0, 0};
    float by_row = 0.0f;
    if (BWD) {
      by_key = *reinterpret_cast<const f32x4_t*>(&scratch->notes.other[4 * gr]);
      by_row = scratch->notes.factor[16 + c];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool below = 4 * gr + r > c;
      const float x0 = d00[r] * n.factor[0][r] * rn0 * pow2(n.G(0, r), n.Gc[0]);
      const float x1 = d11[r] * n.factor[1][r] * rn1 * pow2(n.G(1, r), n.Gc[1]);
      a00[r] = below ? x0 : 0.0f;
      a11[r] = below ? x1 : 0.0f;
      a10[r] = BWD ? d10[r] * by_key[r] * by_row * pow2(n.Gc[1], n.G(0, r))           // row 16 + lane%16, column 4g + r
                   : d10[r] * n.factor[1][r] * rn0 * pow2(n.G(1, r), n.Gc[0]);        // row 16 + 4g + r, column lane%16
    }
    solve_blocks(scratch, a00, a11, lane);
    const f32x4_t zero = {0, 0, 0, 0};
    if (!BWD) {
      // rows of T as operands; T10^T = -T0^T (A10^T T1^T) comes out as the operand's own layout
      const f32x4_t row1 = square_row(scratch->t[1], lane);
      const f32x4_t t10 = square_product(square_column(scratch->t[0], lane), square_product(a10, row1));
      put_triangle<3>(at + B::kT, 0, lane, square_row(scratch->t[0], lane), zero);
      put_triangle<3>(at + B::kT, 1, lane, -t10, row1);
    } else {
      // rows of T^T: columns of T.  T10 = -T1 (A10 T0)
      const f32x4_t col0 = square_column(scratch->t[0], lane);
      const f32x4_t t10 = square_product(square_row(scratch->t[1], lane), square_product(a10, col0));
      put_triangle<3>(at + B::kT, 0, lane, col0, -t10);
      put_triangle<3>(at + B::kT, 1, lane, zero, square_column(scratch->t[1], lane));
    }
  }
};

// Producer of the queries: rows of Q in pieces, M (backward: M^T) and the coefficient kQuery = scale r e^G.
template <class E, int D, bool BWD>
struct QueryProducer {
  typedef ChunkBuffer<E, D, true> B;
  const Args& a;
  const Live lives;
  const Slice& s;
  const __amdgpu_buffer_rsrc_t decays;
  RowTile<E, D> q, k;
  uint32_t live, there, g;  // keys that take part; rows that exist
  uint32_t byte;

  __device__ __forceinline__ QueryProducer(const Args& args, const Slice& slice)
      : a(args), lives(args, slice), s(slice), decays(slice.of_gate(args, args.g)) {}
  __device__ __forceinline__ void fetch(int chunk, int lane) {
    live = lives.bits(byte, chunk);
    there = existing(a.N, chunk);
    q.load(s.of(a.Q, chunk, a.stride_row), a.stride_row, ~0u, lane);
    k.load(s.of(a.K, chunk, a.stride_row), a.stride_row, live, lane);
    g = fetch_gate(a, decays, chunk, live, lane);
  }
  __device__ __forceinline__ void begin(int chunk, int next, int lane) {
    byte = lives.fetch(chunk, lane);
    fetch(chunk, lane);
    byte = lives.fetch(next, lane);
  }
  __device__ __forceinline__ void make(int next, int after, unsigned char* at, Notes* n, int lane) {
    const int c = lane & 15, gr = lane >> 4;
    float* coef = reinterpret_cast<float*>(at + B::kCoef);
    const float rq0 = a.scale * inverse_norm(dots(q, 0, q, 0), 0, a.eps, there, lane);
    const float rq1 = a.scale * inverse_norm(dots(q, 1, q, 1), 1, a.eps, there, lane);
    const float rk0 = inverse_norm(dots(k, 0, k, 0), 0, a.eps, live, lane);
    const float rk1 = inverse_norm(dots(k, 1, k, 1), 1, a.eps, live, lane);
    q.put(at + B::kQ, lane);
    const Sum G = scan_decays(__uint_as_float(g), lane);
    // forward: rows j (keys), columns i (queries); backward: rows i, columns j
    const f32x4_t d00 = BWD ? dots(q, 0, k, 0) : dots(k, 0, q, 0), d11 = BWD ? dots(q, 1, k, 1) : dots(k, 1, q, 1),
                  d10 = BWD ? dots(q, 1, k, 0) : dots(k, 0, q, 1);
    if (lane < 32) {
      n->hi[lane] = G.hi;
      n->lo[lane] = G.lo;
      n->factor[lane] = BWD ? (lane < 16 ? rq0 : rq1) : (lane < 16 ? rk0 : rk1);  // of the rows of the results
      coef[B::kQuery + lane] = (lane < 16 ? rq0 : rq1) * pow2(G);
    }
    if (next >= 0 && next < a.chunks) {
      fetch(next, lane);
      byte = lives.fetch(after, lane);
    }
    wave_fence();
    // rows o = 4g + r, columns lane%16: keys and queries, or queries and keys
    const Noted o(*n, lane);
    f32x4_t m00, m11, m10;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 4 * gr + r;
      const float x0 = d00[r] * o.factor[0][r] * (BWD ? rk0 : rq0) * (BWD ? pow2(o.G(0, r), o.Gc[0]) : pow2(o.Gc[0], o.G(0, r)));
      const float x1 = d11[r] * o.factor[1][r] * (BWD ? rk1 : rq1) * (BWD ? pow2(o.G(1, r), o.Gc[1]) : pow2(o.Gc[1], o.G(1, r)));
      const bool in = BWD ? row >= c : row <= c;
      m00[r] = in ? x0 : 0.0f;
      m11[r] = in ? x1 : 0.0f;
      m10[r] = BWD ? d10[r] * o.factor[1][r] * rk0 * pow2(o.G(1, r), o.Gc[0])
                   : d10[r] * o.factor[0][r] * rq1 * pow2(o.Gc[1], o.G(0, r));
    }
    const f32x4_t zero = {0, 0, 0, 0};
    put_triangle<3>(at + B::kM, 0, lane, m00, BWD ? m10 : zero);
    put_triangle<3>(at + B::kM, 1, lane, BWD ? zero : m10, m11);
  }
};

// Rows of V or dO in the layout of a result: column `col`, tokens 16 tt + 4g + r.
template <class E>
struct ColumnTile {
  typename E::One x[2][4];
  // r: from the chunk's first row on
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t stride, uint32_t live, int col, int lane) {
    const uint32_t first = 4 * (lane >> 4) * stride + col * E::kBytes;
    const uint32_t of_lane = live >> (4 * (lane >> 4));
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[tt][i] = E::load_one(r, offset_if(of_lane, 16 * tt + i, first + (16 * tt + i) * stride));
  }
  // (kept as loaded, 32 bits each, by the empty statement: the compiler would pack 16-bit values in pairs, and wait for them,
  // right behind the loads)
  __device__ __forceinline__ f32x4_t tile(int tt) const {
    f32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = x[tt][i];
      asm("" : "+v"(w));
      r[i] = E::value(w);
    }
    return r;
  }
};

// 16 columns of a state: rows 16 dt + 4g + r, column lane%16 of the wave's; and its pieces, by blocks of 32 rows.
template <int D>
struct StateColumns {
  static constexpr int kTiles = D / 16, kBlocks = D < 32 ? 1 : D / 32;
  f32x4_t s[kBlocks * 2];
  Pieces<3> p[kBlocks];
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t of(const float* state) {  // [D][D]; nullptr: loads bring zeros
    return buffer(state, state == nullptr ? 0 : D * D * 4);
  }
  __device__ __forceinline__ void load(const float* from, int col, int lane) {
    const __amdgpu_buffer_rsrc_t r = of(from);
    const uint32_t first = (4 * (lane >> 4) * D + col) * 4;
#pragma unroll
    for (int dt = 0; dt < 2 * kBlocks; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[dt][i] = dt < kTiles ? __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, first + (16 * dt + i) * D * 4, 0, 0)) : 0.0f;
  }
  __device__ __forceinline__ void unit(int col, int lane) {
#pragma unroll
    for (int dt = 0; dt < 2 * kBlocks; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[dt][i] = 16 * dt + 4 * (lane >> 4) + i == col ? 1.0f : 0.0f;
  }
  __device__ __forceinline__ void store(float* to, int col, int lane) const {
    const __amdgpu_buffer_rsrc_t r = of(to);
    const uint32_t first = (4 * (lane >> 4) * D + col) * 4;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s[dt][i]), r, first + (16 * dt + i) * D * 4, 0, 0);
  }
  template <int OTHER>
  __device__ __forceinline__ void cut_all() {
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) p[kb] = cut<OTHER>(s[2 * kb], s[2 * kb + 1]);
  }
};

// Row 16 dt + lane%16 of a state [D][D] as an operand with the depth in slot order (see Rows).
template <int D>
struct StateRows {
  static constexpr int kBlocks = D < 32 ? 1 : D / 32;
  f32x4_t lo[kBlocks], hi[kBlocks];
  __device__ __forceinline__ void load(const float* from, int dt, int lane) {
    const float* p = from + (16 * dt + (lane & 15)) * D + 4 * (lane >> 4);
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      lo[kb] = *reinterpret_cast<const f32x4_t*>(p + 32 * kb);
      hi[kb] = D < 32 ? f32x4_t{0, 0, 0, 0} : *reinterpret_cast<const f32x4_t*>(p + 32 * kb + (D < 32 ? 0 : 16));
    }
  }
};

// S <- M S + R (TRANSPOSED: M^T S + R), cut.
template <int D, bool TRANSPOSED>
__device__ __forceinline__ void advance(StateColumns<D>& S, const float* M, const float* R, int col, int lane) {
  S.load(R, col, lane);
#pragma unroll
  for (int dt = 0; dt < StateColumns<D>::kTiles; ++dt) {
    if (TRANSPOSED) {
      StateColumns<D> m;
      m.load(M, 16 * dt + (lane & 15), lane);
#pragma unroll
      for (int kb = 0; kb < S.kBlocks; ++kb) S.s[dt] = mul(cut<3>(m.s[2 * kb], m.s[2 * kb + 1]), S.p[kb], S.s[dt]);
    } else {
      StateRows<D> m;
      m.load(M, dt, lane);
#pragma unroll
      for (int kb = 0; kb < S.kBlocks; ++kb) S.s[dt] = mul(cut<3>(m.lo[kb], m.hi[kb]), S.p[kb], S.s[dt]);
    }
  }
  S.template cut_all<3>();
}

// A pair of result tiles (tokens 16 tt + 4g + r, column `col`) into the rows of a chunk [32][D].
template <int D>
__device__ __forceinline__ void store_rows(float* to, const f32x4_t (&x)[2], int col, int lane) {
  const __amdgpu_buffer_rsrc_t r = buffer(to, kChunk * D * 4);
  const uint32_t first = (4 * (lane >> 4) * D + col) * 4;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[tt][i]), r, first + (16 * tt + i) * D * 4, 0, 0);
}

// S += X w: X the columns of the chunk's rows at `rows`, w a chunk's rows in pieces; two tiles of S at a time.
template <class R, int D>
__device__ __forceinline__ void add_outer(StateColumns<D>& S, const unsigned char* rows, const Pieces<3>& w, int lane) {
  if constexpr (D == 16) {
    S.s[0] = mul(R::column_operand(rows, 0, lane), w, S.s[0]);
  } else {
#pragma unroll
    for (int dt = 0; dt < S.kTiles; dt += 2) {
      const decltype(R::column_operand(rows, 0, lane)) x[2] = {R::column_operand(rows, dt, lane), R::column_operand(rows, dt + 1, lane)};
      f32x4_t c[2] = {S.s[dt], S.s[dt + 1]};
      mul_left(x, w, c);
      S.s[dt] = c[0];
      S.s[dt + 1] = c[1];
    }
  }
}
// c[tt] += (rows 16 tt ... of the chunk's rows at `rows`) S; TRANSPOSED: of the same product's transpose
template <class R, int D, bool TRANSPOSED>
__device__ __forceinline__ void add_rows_times(const unsigned char* rows, const StateColumns<D>& S, f32x4_t (&c)[2], int lane) {
#pragma unroll
  for (int kb = 0; kb < S.kBlocks; ++kb) {
    const decltype(R::row_operand(rows, 0, kb, lane)) x[2] = {R::row_operand(rows, 0, kb, lane), R::row_operand(rows, 1, kb, lane)};
    if constexpr (TRANSPOSED) mul_right(S.p[kb], x, c);
    else mul_left(x, S.p[kb], c);
  }
}

__device__ __forceinline__ f32x4_t by_rows(const float* coef, int tt, int lane) {
  return *reinterpret_cast<const f32x4_t*>(coef + 16 * tt + 4 * (lane >> 4));
}

}  // namespace delta
}  // namespace cotten
