// The waves of the chunked kernels of the gated delta rule (see cotten_delta_core.h for the formulas): two producers that
// make what a chunk needs besides the state, and consumers that carry 16 columns of the state each.
#pragma once
#include "cotten_delta_core.h"

namespace cotten {
namespace delta {

// One chunk's place in LDS.  The producers fill one while the consumers read the other.
template <class E, int D>
struct ChunkBuffer {
  typedef Rows<D, E::kPieces> R;
  static constexpr int kK = 0, kQ = R::kBytes, kT = 2 * R::kBytes, kM = kT + kTriangleBytes, kCoef = kM + kTriangleBytes;
  static constexpr int kBytes = kCoef + (5 * kChunk + 4) * 4;
  // coefficients by token: four columns, and e^(G_C) behind them
  enum { kBeta = 0, kReadK = kChunk, kWriteK = 2 * kChunk, kQuery = 3 * kChunk, kAdjoint = 4 * kChunk, kWhole = 5 * kChunk };
};

// Producer of the keys: rows of K in pieces, T (backward: T^T), and the coefficients
//     kReadK  r e^G (what K S is multiplied with)     kWriteK  r e^(G_C - G)     kAdjoint  -beta e^G r (backward)
template <class E, int D, bool BWD>
struct KeyProducer {
  typedef ChunkBuffer<E, D> B;
  RowTile<E, D> k;
  uint32_t live;
  int byte;
  float g, beta;

  __device__ __forceinline__ void gates(const Args& a, const Slice& s, int chunk, int lane) {
    const int t = kChunk * chunk + (lane & 31);
    const bool on = (live >> (lane & 31)) & 1u;
    g = on ? a.g[s.gates + static_cast<long long>(t) * a.gate_row] : 0.0f;
    beta = on ? a.beta[s.gates + static_cast<long long>(t) * a.gate_row] : 0.0f;
  }
  __device__ __forceinline__ void begin(const Args& a, const Slice& s, __amdgpu_buffer_rsrc_t K, int chunk, int next, int lane) {
    live = live_of(fetch_live(s, a.N, chunk, lane));
    k.load(K, a.stride_row, chunk, live, lane);
    gates(a, s, chunk, lane);
    byte = next >= 0 ? fetch_live(s, a.N, next, lane) : 0;
  }
  // makes `chunk` and begins the loads of `next` (-1: none) and of the mask of `after`
  __device__ __forceinline__ void make(const Args& a, const Slice& s, __amdgpu_buffer_rsrc_t K, int next, int after,
                                       unsigned char* at, Scratch* scratch, int lane) {
    const int c = lane & 15, gr = lane >> 4;
    float* coef = reinterpret_cast<float*>(at + B::kCoef);
    const float rn0 = k.inverse_norm(0, a.eps, live, lane), rn1 = k.inverse_norm(1, a.eps, live, lane);
    k.put(at + B::kK, lane);
    const double G = scan_decays(g, (live >> (lane & 31)) & 1u, lane);
    const double G_end = __shfl(G, 31);
    // k_i . k_j: backward keeps the lower block as its transpose, see below
    const f32x4_t d00 = dots(k, 0, k, 0), d11 = dots(k, 1, k, 1), d10 = BWD ? dots(k, 0, k, 1) : dots(k, 1, k, 0);
    if (lane < 32) {
      const float r = lane < 16 ? rn0 : rn1, eG = pow2(G);
      scratch->notes.G[lane] = G;
      scratch->notes.rk[lane] = r;
      scratch->notes.beta[lane] = beta;
      coef[B::kBeta + lane] = beta;
      coef[B::kReadK + lane] = r * eG;
      coef[B::kWriteK + lane] = r * pow2(G_end - G);
      if (BWD) coef[B::kAdjoint + lane] = -beta * eG * r;
      if (lane == 31) coef[B::kWhole] = eG;
    }
    // the next chunk's rows, while this one is worked on
    if (next >= 0) {
      live = live_of(byte);
      k.load(K, a.stride_row, next, live, lane);
      gates(a, s, next, lane);
      byte = after >= 0 ? fetch_live(s, a.N, after, lane) : 0;
    }
    wave_fence();
    const Notes& n = scratch->notes;
    f32x4_t a00, a11, a10;
    const double Gc0 = n.G[c], Gc1 = n.G[16 + c];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * gr + r;
      const float f0 = n.beta[i] * n.rk[i], f1 = n.beta[16 + i] * n.rk[16 + i];
      a00[r] = i > c ? d00[r] * f0 * rn0 * pow2(n.G[i] - Gc0) : 0.0f;
      a11[r] = i > c ? d11[r] * f1 * rn1 * pow2(n.G[16 + i] - Gc1) : 0.0f;
      if (!BWD) a10[r] = d10[r] * f1 * rn0 * pow2(n.G[16 + i] - Gc0);            // row 16+i, column c
      else a10[r] = d10[r] * (n.beta[16 + c] * rn1) * n.rk[i] * pow2(Gc1 - n.G[i]);  // row 16+c, column i
    }
    solve_blocks(scratch, a00, a11, lane);
    const f32x4_t zero = {0, 0, 0, 0};
    if (!BWD) {
      // rows of T as operands; T10^T = -T0^T (A10^T T1^T) comes out as the operand's own layout
      const f32x4_t row1 = square_row(scratch->t[1], lane);
      const f32x4_t t10 = square_product(square_column(scratch->t[0], lane), square_product(a10, row1));
      put_triangle(at + B::kT, 0, lane, square_row(scratch->t[0], lane), zero);
      put_triangle(at + B::kT, 1, lane, -t10, row1);
    } else {
      // rows of T^T: columns of T.  T10 = -T1 (A10 T0)
      const f32x4_t col0 = square_column(scratch->t[0], lane);
      const f32x4_t t10 = square_product(square_row(scratch->t[1], lane), square_product(a10, col0));
      put_triangle(at + B::kT, 0, lane, col0, -t10);
      put_triangle(at + B::kT, 1, lane, zero, square_column(scratch->t[1], lane));
    }
  }
};

// Producer of the queries: rows of Q in pieces, M (backward: M^T) and the coefficient kQuery = scale r e^G.
template <class E, int D, bool BWD>
struct QueryProducer {
  typedef ChunkBuffer<E, D> B;
  RowTile<E, D> q, k;
  uint32_t live, there;  // keys that take part; rows that exist
  int byte;
  float g;

  __device__ __forceinline__ void fetch(const Args& a, const Slice& s, __amdgpu_buffer_rsrc_t Q, __amdgpu_buffer_rsrc_t K,
                                        int chunk, int lane) {
    there = existing(a.N, chunk);
    q.load(Q, a.stride_row, chunk, there, lane);
    k.load(K, a.stride_row, chunk, live, lane);
    const int t = kChunk * chunk + (lane & 31);
    g = ((live >> (lane & 31)) & 1u) ? a.g[s.gates + static_cast<long long>(t) * a.gate_row] : 0.0f;
  }
  __device__ __forceinline__ void begin(const Args& a, const Slice& s, __amdgpu_buffer_rsrc_t Q, __amdgpu_buffer_rsrc_t K,
                                        int chunk, int next, int lane) {
    live = live_of(fetch_live(s, a.N, chunk, lane));
    fetch(a, s, Q, K, chunk, lane);
    byte = next >= 0 ? fetch_live(s, a.N, next, lane) : 0;
  }
  __device__ __forceinline__ void make(const Args& a, const Slice& s, __amdgpu_buffer_rsrc_t Q, __amdgpu_buffer_rsrc_t K,
                                       int next, int after, unsigned char* at, Notes* n, int lane) {
    const int c = lane & 15, gr = lane >> 4;
    float* coef = reinterpret_cast<float*>(at + B::kCoef);
    const float rq0 = a.scale * q.inverse_norm(0, a.eps, there, lane), rq1 = a.scale * q.inverse_norm(1, a.eps, there, lane);
    const float rk0 = k.inverse_norm(0, a.eps, live, lane), rk1 = k.inverse_norm(1, a.eps, live, lane);
    q.put(at + B::kQ, lane);
    const double G = scan_decays(g, (live >> (lane & 31)) & 1u, lane);
    // forward: rows j (keys), columns i (queries); backward: rows i, columns j
    const f32x4_t d00 = BWD ? dots(q, 0, k, 0) : dots(k, 0, q, 0), d11 = BWD ? dots(q, 1, k, 1) : dots(k, 1, q, 1),
                  d10 = BWD ? dots(q, 1, k, 0) : dots(k, 0, q, 1);
    if (lane < 32) {
      n->G[lane] = G;
      n->rk[lane] = BWD ? (lane < 16 ? rq0 : rq1) : (lane < 16 ? rk0 : rk1);  // of the rows of the results
      coef[B::kQuery + lane] = (lane < 16 ? rq0 : rq1) * pow2(G);
    }
    if (next >= 0) {
      live = live_of(byte);
      fetch(a, s, Q, K, next, lane);
      byte = after >= 0 ? fetch_live(s, a.N, after, lane) : 0;
    }
    wave_fence();
    f32x4_t m00, m11, m10;
    const double Gc0 = n->G[c], Gc1 = n->G[16 + c];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int o = 4 * gr + r;  // the other index: c and o are query and key, or key and query
      const double Go0 = n->G[o], Go1 = n->G[16 + o];
      const float fo0 = n->rk[o], fo1 = n->rk[16 + o];
      if (!BWD) {
        m00[r] = o <= c ? d00[r] * fo0 * rq0 * pow2(Gc0 - Go0) : 0.0f;
        m11[r] = o <= c ? d11[r] * fo1 * rq1 * pow2(Gc1 - Go1) : 0.0f;
        m10[r] = d10[r] * fo0 * rq1 * pow2(Gc1 - Go0);
      } else {
        m00[r] = o >= c ? d00[r] * fo0 * rk0 * pow2(Go0 - Gc0) : 0.0f;
        m11[r] = o >= c ? d11[r] * fo1 * rk1 * pow2(Go1 - Gc1) : 0.0f;
        m10[r] = d10[r] * fo1 * rk0 * pow2(Go1 - Gc0);
      }
    }
    const f32x4_t zero = {0, 0, 0, 0};
    put_triangle(at + B::kM, 0, lane, m00, BWD ? m10 : zero);
    put_triangle(at + B::kM, 1, lane, BWD ? zero : m10, m11);
  }
};

// Rows of V or dO in the layout of a result: column `col`, tokens 16 tt + 4g + r.
template <class E>
struct ColumnTile {
  float x[2][4];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t stride, int chunk, uint32_t live, int col, int lane) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 16 * tt + 4 * (lane >> 4) + i;
        const uint32_t off = static_cast<uint32_t>(kChunk * chunk + row) * stride + col * E::kBytes;
        x[tt][i] = E::load_one(r, ((live >> row) & 1u) ? off : kNowhere);
      }
  }
  __device__ __forceinline__ f32x4_t tile(int tt) const { return f32x4_t{x[tt][0], x[tt][1], x[tt][2], x[tt][3]}; }
};

// 16 columns of a state: rows 16 dt + 4g + r, column lane%16 of the wave's; and its pieces, by blocks of 32 rows.
template <int D>
struct StateColumns {
  static constexpr int kTiles = D / 16, kBlocks = D < 32 ? 1 : D / 32;
  f32x4_t s[kBlocks * 2];
  Pieces<3> p[kBlocks];
  __device__ __forceinline__ void load(const float* from, int col, int lane) {  // from: [D][D] or nullptr
#pragma unroll
    for (int dt = 0; dt < 2 * kBlocks; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        s[dt][r] = dt < kTiles && from != nullptr ? from[(16 * dt + 4 * (lane >> 4) + r) * D + col] : 0.0f;
  }
  __device__ __forceinline__ void store(float* to, int col, int lane) const {
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) to[(16 * dt + 4 * (lane >> 4) + r) * D + col] = s[dt][r];
  }
  __device__ __forceinline__ void cut_all() {
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) p[kb] = cut(s[2 * kb], s[2 * kb + 1]);
  }
};

__device__ __forceinline__ f32x4_t by_rows(const float* coef, int tt, int lane) {
  return *reinterpret_cast<const f32x4_t*>(coef + 16 * tt + 4 * (lane >> 4));
}

}  // namespace delta
}  // namespace cotten
