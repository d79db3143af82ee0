// Backward of the gated delta rule (cotten_delta_core.h has the forward's formulas).  With the gradient dS' of the state
// after a chunk:
//
//     dU = scale M^T dO + e^(G_C - G) (K^ dS')          Z = T^T dU            dV = beta Z
//     dS = e^(G_C) dS' + scale Q^^T (e^G dO) - K^^T (beta e^G Z)
//
// goes from chunk to chunk in reverse order, column by column as the forward does (chunk_adjoint_kernel).  The rest needs
// the states on both sides of a chunk and no other chunk (chunk_gradient_kernel): with D_ij = e^(G_i - G_j),
//
//     dq^ = scale (e^G (dO S^T) + (D . dO U^T) K^)                                   (j <= i)
//     p   = -e^G (Z S^T) - (D . Z U^T) K^                                            (j < i)
//     w   = e^(G_C - G) (U dS'^T) + scale (D . dO U^T)^T Q^ - (beta D . Z U^T)^T K^
//     dk^ = beta p + w      dbeta = Z . v + k^ . p      dx = (dx^ - x^ (x^ . dx^)) / r(x)
//     dg_t = sum_{i >= t > j} F_ij + sum_{i >= t} r_i + sum_{j < t} c_j + e^(G_C) <S, dS'>
//         F_ij = scale D_ij (dO U^T)_ij q^_i . k^_j - beta_i D_ij (Z U^T)_ij k^_i . k^_j
//         r_i  = scale e^(G_i) q^_i . (dO S^T)_i - beta_i e^(G_i) k^_i . (Z S^T)_i      c_j = e^(G_C - G_j) k^_j . (U dS'^T)_j
//
// (a decay counts for what was written before it and read from it on.  The same sums follow from the products q^ . dq^,
// k^ . dk^ of whole rows, with fewer operations; but there the pairs on one side of t cancel, and strong decays
// would leave the rounding errors of terms that are not small.)
#include "cotten_delta_chunk.h"
#include "cotten_delta_launch.h"
#include "cotten_launch.h"

namespace cotten {
namespace delta {
namespace {

extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

template <int D>
constexpr int kConsumers = D / 16 < 4 ? D / 16 : 4;

// The forward's walk in reverse: two producers, and waves with 16 columns of dS each.  Writes dS' and Z for the second
// kernel, and dV.
template <class E, int D>
__global__ __launch_bounds__(64 * (kConsumers<D> + 2)) void chunk_adjoint_kernel(Args a) {
  typedef ChunkBuffer<E, D> B;
  typedef typename B::R R;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int kGroups = D / 16 / kConsumers<D>;
  const int slice = blockIdx.x / kGroups, group = blockIdx.x % kGroups;
  const Slice s(a, slice, D * E::kBytes);
  Scratch* scratch = reinterpret_cast<Scratch*>(smem + 2 * B::kBytes);
  Notes* notes = reinterpret_cast<Notes*>(scratch + 1);
  const __amdgpu_buffer_rsrc_t K = s.of(a.K);
  const int last = a.chunks - 1;

  if (wave == 0) {
    KeyProducer<E, D, true> producer;
    producer.begin(a, s, K, last, last - 1, lane);  // (-1: none)
    for (int c = last; c >= -1; --c) {
      if (c >= 0) producer.make(a, s, K, c - 1, c > 0 ? c - 2 : -1, smem + (c & 1) * B::kBytes, scratch, lane);
      __syncthreads();
    }
  } else if (wave == 1) {
    const __amdgpu_buffer_rsrc_t Q = s.of(a.Q);
    QueryProducer<E, D, true> producer;
    producer.begin(a, s, Q, K, last, last - 1, lane);
    for (int c = last; c >= -1; --c) {
      if (c >= 0) producer.make(a, s, Q, K, c - 1, c > 0 ? c - 2 : -1, smem + (c & 1) * B::kBytes, notes, lane);
      __syncthreads();
    }
  } else {
    const __amdgpu_buffer_rsrc_t G = s.of(a.dO), dV = s.of(a.dV);
    const int tile = group * kConsumers<D> + wave - 2, col = 16 * tile + (lane & 15);
    const long long state = static_cast<long long>(slice) * D * D;
    StateColumns<D> dS;
    dS.load(a.dfinal_state == nullptr ? nullptr : a.dfinal_state + state, col, lane);
    dS.cut_all();
    ColumnTile<E> g;
    g.load(G, a.stride_row, last, existing(a.N, last), col, lane);
    uint32_t live = live_of(fetch_live(s, a.N, last, lane));
    __syncthreads();
    for (int c = last; c >= 0; --c) {
      const unsigned char* at = smem + (c & 1) * B::kBytes;
      const float* coef = reinterpret_cast<const float*>(at + B::kCoef);
      const long long chunk = static_cast<long long>(slice) * a.chunks + c;
      dS.store(a.dstates + chunk * D * D, col, lane);
      const int byte = c > 0 ? fetch_live(s, a.N, c - 1, lane) : 0;
      const Pieces<E::kPieces> up = cut_elements<E>(g.tile(0), g.tile(1));
      const Pieces<3> write = cut(g.tile(0) * by_rows(coef + B::kQuery, 0, lane), g.tile(1) * by_rows(coef + B::kQuery, 1, lane));
      if (c > 0) g.load(G, a.stride_row, c - 1, ~0u, col, lane);
      f32x4_t z[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        f32x4_t p = {0, 0, 0, 0};
#pragma unroll
        for (int kb = 0; kb < dS.kBlocks; ++kb) p = mul(R::row_operand(at + B::kK, tt, kb, lane), dS.p[kb], p);
        z[tt] = mul(triangle_operand(at + B::kM, tt, lane), up, by_rows(coef + B::kWriteK, tt, lane) * p);
      }
      const Pieces<3> y = cut(z[0], z[1]);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) z[tt] = mul(triangle_operand(at + B::kT, tt, lane), y, f32x4_t{0, 0, 0, 0});
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const f32x4_t beta = by_rows(coef + B::kBeta, tt, lane);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = 16 * tt + 4 * (lane >> 4) + r, row = kChunk * c + t;
          a.rows_z[(chunk * kChunk + t) * D + col] = z[tt][r];
          E::store_one(dV, row < a.N ? static_cast<uint32_t>(row) * a.stride_row + col * E::kBytes : kNowhere,
                       ((live >> t) & 1u) ? beta[r] * z[tt][r] : 0.0f);
        }
      }
      const float whole = coef[B::kWhole];
      const Pieces<3> w = cut(z[0] * by_rows(coef + B::kAdjoint, 0, lane), z[1] * by_rows(coef + B::kAdjoint, 1, lane));
#pragma unroll
      for (int dt = 0; dt < dS.kTiles; ++dt) {
        dS.s[dt] = mul(R::column_operand(at + B::kQ, dt, lane), write, dS.s[dt] * whole);
        dS.s[dt] = mul(R::column_operand(at + B::kK, dt, lane), w, dS.s[dt]);
      }
      dS.cut_all();
      live = live_of(byte);
      __syncthreads();
    }
    if (a.dinitial_state != nullptr) dS.store(a.dinitial_state + state, col, lane);
  }
}

// One chunk: a wave has 16 columns (of d_h as the index of q and k) of every result.  Results are computed transposed, so
// a lane has four columns of one token: factors by token are one value, stores are whole pieces of a row.
template <class E, int D>
struct GradientLds {
  typedef Rows<D, E::kPieces> R;
  typedef Rows<D, 3> R3;
  static constexpr int kK = 0, kQ = R::kBytes, kG = 2 * R::kBytes, kU = 3 * R::kBytes, kZ = kU + R3::kBytes;
  static constexpr int kTriangles = kZ + R3::kBytes, kSums = kTriangles + 4 * kTriangleBytes;
  static constexpr int kWaves = D / 16;
  // per wave: q^ . dq^, k^ . p, k^ . w, Z . v, r and c by token, <S, dS'>
  static constexpr int kOfWave = 6 * kChunk + 4;
  static constexpr int kPairs = kSums + kWaves * kOfWave * 4;  // sums of F by token, of its two terms
  static constexpr int kNotes = kPairs + 2 * kChunk * 4, kBytes = kNotes + 2 * kChunk * 4;
};

// Rows 16 tt .. of a chunk into LDS; returns 1/r of row lane%16 of them.
template <class E, int D>
__device__ __forceinline__ float stage(unsigned char* at, __amdgpu_buffer_rsrc_t r, uint32_t stride, int first, uint32_t live,
                                       int tt, float eps, int lane) {
  typedef Rows<D, E::kPieces> R;
  const int row = 16 * tt + (lane & 15), g = lane >> 4;
  const bool on = ((live >> row) & 1u) != 0;
  const uint32_t off = static_cast<uint32_t>(first + row) * stride + g * 8 * E::kBytes;
  float ss = 0.0f;
#pragma unroll
  for (int kb = 0; kb < R::kBlocks; ++kb) {
    const typename E::Raw raw = E::load(r, on && (D >= 32 || g * 8 < D) ? off + kb * 32 * E::kBytes : kNowhere);
    float x[8];
    E::unpack(raw, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
    R::put(at, row, kb, g, E::pieces(raw));
  }
  ss += __shfl_xor(ss, 16);
  ss += __shfl_xor(ss, 32);
  return on ? __builtin_amdgcn_rsqf(ss + eps) : 0.0f;
}

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

__device__ __forceinline__ float over_groups(float x) {  // sum over the four lanes with the same lane%16
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// sum over i >= t > j of F, t = 0 ... 31, from its tiles (i tile, j tile) (0,0), (1,1), (1,0) as results (row i, column j).
__device__ __forceinline__ void pair_sums(f32x4_t f00, f32x4_t f11, f32x4_t f10, float* to, int lane) {
  const int c = lane & 15, g = lane >> 4;
  // sums over rows from each row on: of the tile's own lane, then of the lane groups behind
  auto suffix = [&](f32x4_t f) {
#pragma unroll
    for (int r = 2; r >= 0; --r) f[r] += f[r + 1];
    const float own = f[0];
    float behind = 0.0f;
#pragma unroll
    for (int d = 1; d < 4; ++d) {
      const float x = __shfl(own, (lane + 16 * d) & 63);
      behind += g + d < 4 ? x : 0.0f;
    }
    return f + behind;
  };
  const f32x4_t s00 = suffix(f00), s11 = suffix(f11), s10 = suffix(f10);
  const float all10 = __shfl(s10[0], c);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = 4 * g + r;
    float x = c < t ? s00[r] + all10 : 0.0f, y = s10[r] + (c < t ? s11[r] : 0.0f);
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
      x += __shfl_xor(x, m);
      y += __shfl_xor(y, m);
    }
    if (c == 0) {
      to[t] = x;
      to[16 + t] = y;
    }
  }
}

template <class E, int D>
__global__ __launch_bounds__(64 * (D / 16)) void chunk_gradient_kernel(Args a) {
  typedef GradientLds<E, D> L;
  typedef typename L::R R;
  typedef typename L::R3 R3;
  constexpr int kWaves = L::kWaves;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, gr = lane >> 4;
  const long long chunk = blockIdx.x;
  const int slice = static_cast<int>(chunk / a.chunks), c = static_cast<int>(chunk - static_cast<long long>(slice) * a.chunks);
  const Slice s(a, slice, D * E::kBytes);
  const uint32_t live = live_of(fetch_live(s, a.N, c, lane)), there = existing(a.N, c);
  float* rk = reinterpret_cast<float*>(smem + L::kNotes);
  float* rq = rk + kChunk;
  const __amdgpu_buffer_rsrc_t Q = s.of(a.Q), K = s.of(a.K), V = s.of(a.V);

  StateRows<D> before, after;
  before.load(a.states + chunk * D * D, wave, lane);
  after.load(a.dstates + chunk * D * D, wave, lane);
  const bool on = (live >> (lane & 31)) & 1u;
  const long long gate = s.gates + (static_cast<long long>(kChunk) * c + (lane & 31)) * a.gate_row;
  const float g = on ? a.g[gate] : 0.0f, beta = on ? a.beta[gate] : 0.0f;
  // K, Q, dO, U, Z, half a chunk at a time, dealt to the waves
  for (int item = wave; item < 10; item += kWaves) {
    const int tt = item & 1;
    if (item < 2) {
      const float r = stage<E, D>(smem + L::kK, K, a.stride_row, kChunk * c, live, tt, a.eps, lane);
      if (lane < 16) rk[16 * tt + lane] = r;
    } else if (item < 4) {
      const float r = stage<E, D>(smem + L::kQ, Q, a.stride_row, kChunk * c, there, tt, a.eps, lane);
      if (lane < 16) rq[16 * tt + lane] = r;
    } else if (item < 6) {
      stage<E, D>(smem + L::kG, s.of(a.dO), a.stride_row, kChunk * c, there, tt, 1.0f, lane);
    } else {
      const float* rows = (item < 8 ? a.rows_u : a.rows_z) + chunk * kChunk * D;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(rows), 0, kChunk * D * 4, 0x00020000);
      stage<F32, D>(smem + (item < 8 ? L::kU : L::kZ), r, D * 4, 0, ~0u, tt, 1.0f, lane);
    }
  }
  const double G = scan_decays(g, on, lane), G_end = __shfl(G, 31);
  __syncthreads();

  // the four triangles (query i, key j; both factors of the unit rows of the operand they meet are in them):
  //   0  rows j, columns i:  scale D rk_j (dO U^T)        1  rows i, columns j:  scale D rq_i (dO U^T)
  //   2  rows j, columns i: -D rk_j (Z U^T), j < i        3  rows i, columns j: -beta_i D rk_i (Z U^T), j < i
  for (int job = wave; job < 4; job += kWaves) {
    const bool by_i = (job & 1) != 0;  // rows are i
    const unsigned char* left = smem + (job < 2 ? L::kG : L::kZ);
    f32x4_t m[3] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};  // (i tile, j tile): (0,0), (1,1), (1,0)
#pragma unroll
    for (int kb = 0; kb < R::kBlocks; ++kb) {
      const Pieces<3> u0 = R3::row_operand(smem + L::kU, 0, kb, lane), u1 = R3::row_operand(smem + L::kU, 1, kb, lane);
      auto products = [&](auto x0, auto x1) {
        if (by_i) {
          m[0] = mul(x0, u0, m[0]);
          m[1] = mul(x1, u1, m[1]);
          m[2] = mul(x1, u0, m[2]);
        } else {
          m[0] = mul(u0, x0, m[0]);
          m[1] = mul(u1, x1, m[1]);
          m[2] = mul(u0, x1, m[2]);
        }
      };
      if (job < 2) products(R::row_operand(left, 0, kb, lane), R::row_operand(left, 1, kb, lane));
      else products(R3::row_operand(left, 0, kb, lane), R3::row_operand(left, 1, kb, lane));
    }
    const double Gc[2] = {__shfl(G, c16), __shfl(G, 16 + c16)};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int o = 4 * gr + r;
      const double Go[2] = {__shfl(G, o), __shfl(G, 16 + o)};
      const float* factor = job == 1 ? rq : rk;
      float f[2] = {factor[o], factor[16 + o]};
      if (job < 2) {
        f[0] *= a.scale;
        f[1] *= a.scale;
      } else {
        const float b0 = __shfl(beta, o), b1 = __shfl(beta, 16 + o);
        f[0] *= by_i ? -b0 : -1.0f;
        f[1] *= by_i ? -b1 : -1.0f;
      }
      const bool diagonal = by_i ? (job < 2 ? o >= c16 : o > c16) : (job < 2 ? o <= c16 : o < c16);
      m[0][r] = diagonal ? m[0][r] * f[0] * pow2(by_i ? Go[0] - Gc[0] : Gc[0] - Go[0]) : 0.0f;
      m[1][r] = diagonal ? m[1][r] * f[1] * pow2(by_i ? Go[1] - Gc[1] : Gc[1] - Go[1]) : 0.0f;
      m[2][r] *= by_i ? f[1] * pow2(Go[1] - Gc[0]) : f[0] * pow2(Gc[1] - Go[0]);
    }
    const f32x4_t zero = {0, 0, 0, 0};
    if (by_i) {
      const unsigned char* rows = smem + (job == 1 ? L::kQ : L::kK);
      f32x4_t d00 = zero, d11 = zero, d10 = zero;
#pragma unroll
      for (int kb = 0; kb < R::kBlocks; ++kb) {
        const auto x0 = R::row_operand(rows, 0, kb, lane), x1 = R::row_operand(rows, 1, kb, lane);
        const auto k0 = R::row_operand(smem + L::kK, 0, kb, lane), k1 = R::row_operand(smem + L::kK, 1, kb, lane);
        d00 = mul(x0, k0, d00);
        d11 = mul(x1, k1, d11);
        d10 = mul(x1, k0, d10);
      }
      d00 *= m[0] * rk[c16];
      d11 *= m[1] * rk[16 + c16];
      d10 *= m[2] * rk[c16];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (4 * gr + r <= c16) d00[r] = d11[r] = 0.0f;
      }
      pair_sums(d00, d11, d10, reinterpret_cast<float*>(smem + L::kPairs) + (job >> 1) * kChunk, lane);
    }
    unsigned char* at = smem + L::kTriangles + job * kTriangleBytes;
    put_triangle(at, 0, lane, m[0], by_i ? m[2] : zero);
    put_triangle(at, 1, lane, by_i ? zero : m[2], m[1]);
  }

  // what the states give, tokens in columns
  f32x4_t dq[2], p[2], w[2];
  {
    Pieces<3> S[R::kBlocks];
#pragma unroll
    for (int kb = 0; kb < R::kBlocks; ++kb) S[kb] = cut(before.lo[kb], before.hi[kb]);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      dq[tt] = p[tt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int kb = 0; kb < R::kBlocks; ++kb) {
        dq[tt] = mul(S[kb], R::row_operand(smem + L::kG, tt, kb, lane), dq[tt]);
        p[tt] = mul(S[kb], R3::row_operand(smem + L::kZ, tt, kb, lane), p[tt]);
      }
    }
  }
  float inner = 0.0f;  // <S, dS'> over the wave's columns
#pragma unroll
  for (int kb = 0; kb < R::kBlocks; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) inner += before.lo[kb][r] * after.lo[kb][r] + before.hi[kb][r] * after.hi[kb][r];
  {
    Pieces<3> S[R::kBlocks];
#pragma unroll
    for (int kb = 0; kb < R::kBlocks; ++kb) S[kb] = cut(after.lo[kb], after.hi[kb]);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      w[tt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int kb = 0; kb < R::kBlocks; ++kb) w[tt] = mul(S[kb], R3::row_operand(smem + L::kU, tt, kb, lane), w[tt]);
    }
  }
  const float whole = pow2(G_end);
  inner *= whole;
  f32x4_t q[2], k[2];
  float beta_t[2], rk_t[2], rq_t[2], read[2] = {0.0f, 0.0f}, write[2] = {0.0f, 0.0f};
  uint32_t off[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    const double Gt = __shfl(G, t);
    const float eG = pow2(Gt);
    beta_t[tt] = __shfl(beta, t);
    rk_t[tt] = rk[t];
    rq_t[tt] = rq[t];
    off[tt] = static_cast<uint32_t>(kChunk * c + t) * a.stride_row + (16 * wave + 4 * gr) * E::kBytes;
    q[tt] = E::load_four(Q, ((there >> t) & 1u) ? off[tt] : kNowhere) * rq_t[tt];
    k[tt] = E::load_four(K, ((live >> t) & 1u) ? off[tt] : kNowhere) * rk_t[tt];
    dq[tt] *= a.scale * eG;
    p[tt] *= -eG;
    w[tt] *= pow2(G_end - Gt);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      read[tt] = fmaf(q[tt][r], dq[tt][r], fmaf(beta_t[tt] * k[tt][r], p[tt][r], read[tt]));
      write[tt] = fmaf(k[tt][r], w[tt][r], write[tt]);
    }
  }
  __syncthreads();
  {
    const Pieces<E::kPieces> kc = R::column_operand(smem + L::kK, wave, lane), qc = R::column_operand(smem + L::kQ, wave, lane);
    const unsigned char* at = smem + L::kTriangles;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      dq[tt] = mul(kc, triangle_operand(at, tt, lane), dq[tt]);
      p[tt] = mul(kc, triangle_operand(at + 2 * kTriangleBytes, tt, lane), p[tt]);
      w[tt] = mul(qc, triangle_operand(at + kTriangleBytes, tt, lane), w[tt]);
      w[tt] = mul(kc, triangle_operand(at + 3 * kTriangleBytes, tt, lane), w[tt]);
    }
  }
  // products of a row with its gradients, over all columns
  float* sums = reinterpret_cast<float*>(smem + L::kSums);
  constexpr int kSumsOfWave = L::kOfWave;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    const f32x4_t v = E::load_four(V, ((live >> t) & 1u) ? off[tt] : kNowhere);
    const f32x4_t z = *reinterpret_cast<const f32x4_t*>(a.rows_z + (chunk * kChunk + t) * D + 16 * wave + 4 * gr);
    float qd = 0.0f, kp = 0.0f, kw = 0.0f, zv = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      qd = fmaf(q[tt][r], dq[tt][r], qd);
      kp = fmaf(k[tt][r], p[tt][r], kp);
      kw = fmaf(k[tt][r], w[tt][r], kw);
      zv = fmaf(z[r], v[r], zv);
    }
    qd = over_groups(qd);
    kp = over_groups(kp);
    kw = over_groups(kw);
    zv = over_groups(zv);
    // lane group gr keeps the gr-th of them
    sums[wave * kSumsOfWave + gr * kChunk + t] = gr == 0 ? qd : gr == 1 ? kp : gr == 2 ? kw : zv;
    const float reads = over_groups(read[tt]), writes = over_groups(write[tt]);
    if (gr < 2) sums[wave * kSumsOfWave + (4 + gr) * kChunk + t] = gr == 0 ? reads : writes;
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) inner += __shfl_xor(inner, m);
  if (lane == 0) sums[wave * kSumsOfWave + 6 * kChunk] = inner;
  __syncthreads();
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    float qd = 0.0f, kd = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      qd += sums[i * kSumsOfWave + t];
      kd += beta_t[tt] * sums[i * kSumsOfWave + kChunk + t] + sums[i * kSumsOfWave + 2 * kChunk + t];
    }
    f32x4_t x, y;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[r] = (dq[tt][r] - q[tt][r] * qd) * rq_t[tt];
      y[r] = ((live >> t) & 1u) ? (beta_t[tt] * p[tt][r] + w[tt][r] - k[tt][r] * kd) * rk_t[tt] : 0.0f;
    }
    const uint32_t to = ((there >> t) & 1u) ? off[tt] : kNowhere;
    E::store_four(s.of(a.dQ), to, x);
    E::store_four(s.of(a.dK), to, y);
  }
  if (wave == 0) {
    const int t = lane & 31;
    float kp = 0.0f, zv = 0.0f, reads = 0.0f, writes = 0.0f, end = 0.0f;
    for (int i = 0; i < kWaves; ++i) {
      const float* of = sums + i * kSumsOfWave;
      kp += of[kChunk + t];
      zv += of[3 * kChunk + t];
      reads += of[4 * kChunk + t];
      writes += of[5 * kChunk + t];
      end += of[6 * kChunk];
    }
    const float* pairs = reinterpret_cast<const float*>(smem + L::kPairs);
    writes = __shfl_up(writes, 1, 32);
    if (t == 0) writes = 0.0f;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const float r = __shfl_down(reads, d, 32), w1 = __shfl_up(writes, d, 32);
      if (t + d < 32) reads += r;
      if (t >= d) writes += w1;
    }
    const float x = pairs[t] + pairs[kChunk + t] + reads + writes + end;
    if (lane < 32 && ((there >> t) & 1u)) {
      a.dg[gate] = on ? x : 0.0f;
      a.dbeta[gate] = on ? zv + kp : 0.0f;
    }
  }
}

template <class E, int D>
hipError_t launch(const Args& a, int slices, hipStream_t stream) {
  constexpr int kLds = 2 * ChunkBuffer<E, D>::kBytes + sizeof(Scratch) + sizeof(Notes);
  if (hipError_t err = grant_dynamic_lds(reinterpret_cast<const void*>(chunk_adjoint_kernel<E, D>), kLds); err != hipSuccess) return err;
  chunk_adjoint_kernel<E, D><<<dim3(slices * (D / 16 / kConsumers<D>)), dim3(64 * (kConsumers<D> + 2)), kLds, stream>>>(a);
  if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
  typedef GradientLds<E, D> L;
  static_assert(L::kBytes <= 160 * 1024, "fits the LDS of a compute unit");
  if (hipError_t err = grant_dynamic_lds(reinterpret_cast<const void*>(chunk_gradient_kernel<E, D>), L::kBytes); err != hipSuccess) return err;
  chunk_gradient_kernel<E, D><<<dim3(static_cast<uint32_t>(static_cast<long long>(slices) * a.chunks)), dim3(64 * L::kWaves), L::kBytes, stream>>>(a);
  return hipGetLastError();
}

template <class E>
hipError_t launch_dim(const Args& a, int D, int slices, hipStream_t stream) {
  switch (D) {
    case 16: return launch<E, 16>(a, slices, stream);
    case 32: return launch<E, 32>(a, slices, stream);
    case 64: return launch<E, 64>(a, slices, stream);
    default: return launch<E, 128>(a, slices, stream);
  }
}

}  // namespace

hipError_t launch_backward(const Args& a, int dtype, int D, int slices, hipStream_t stream) {
  return dtype == 0 ? launch_dim<F32>(a, D, slices, stream)
         : dtype == 1 ? launch_dim<Bf16>(a, D, slices, stream)
                      : launch_dim<F16>(a, D, slices, stream);
}

}  // namespace delta
}  // namespace cotten
