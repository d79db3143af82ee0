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
// kernel, and dV.  CARRY: only the gradient of the state before a segment, of segments 1 ...  Bound like the forward's walk,
// and by 24 KB of dS' and Z a chunk (d = 64): 128 x 4 x 200 x 64 bf16 in 40 us, 256 x 2 x 200 x 32 fp32 in 27.
template <class E, int D>
constexpr int kWalkLds = 2 * ChunkBuffer<E, D, true>::kBytes + sizeof(Scratch) + sizeof(Notes);

template <class E, int D, bool CARRY>
__global__ __launch_bounds__(64 * (kConsumers<D> + 2), waves_per_simd(kConsumers<D> + 2, kWalkLds<E, D>)) void chunk_adjoint_kernel(Args a) {
  typedef ChunkBuffer<E, D, true> B;
  typedef typename B::R R;
  const int lane = threadIdx.x & 63, wave = role_of_wave<(kConsumers<D> + 2)>();
  constexpr int kGroups = D / 16 / kConsumers<D>;
  const int unit = blockIdx.x / kGroups, group = blockIdx.x % kGroups;
  const int walked = CARRY ? a.segments - 1 : a.segments;
  const int slice = unit / walked, segment = unit - slice * walked + (CARRY ? 1 : 0);
  const Slice s(a, slice, D * E::kBytes);
  Scratch* scratch = reinterpret_cast<Scratch*>(smem + 2 * B::kBytes);
  Notes* notes = reinterpret_cast<Notes*>(scratch + 1);
  const int first = segment * a.segment_chunks;
  const int last = (first + a.segment_chunks < a.chunks ? first + a.segment_chunks : a.chunks) - 1;

  if (wave == 0) {
    KeyProducer<E, D, true, true> producer(a, s);
    producer.begin(last, last > 0 ? last - 1 : 0, lane);
    for (int c = last; c >= first - 1; --c) {
      if (c >= first) producer.make(c - 1, c > 1 ? c - 2 : 0, smem + (c & 1) * B::kBytes, scratch, lane);
      lds_barrier();
    }
  } else if (wave == 1) {
    QueryProducer<E, D, true> producer(a, s);
    producer.begin(last, last > 0 ? last - 1 : 0, lane);
    for (int c = last; c >= first - 1; --c) {
      if (c >= first) producer.make(c - 1, c > 1 ? c - 2 : 0, smem + (c & 1) * B::kBytes, notes, lane);
      lds_barrier();
    }
  } else {
    const int tile = group * kConsumers<D> + wave - 2, col = 16 * tile + (lane & 15);
    const long long state = static_cast<long long>(slice) * D * D;
    const long long of_segment = static_cast<long long>(slice) * a.segments;
    StateColumns<D> dS;
    if (segment == a.segments - 1) {
      dS.load(a.dfinal_state == nullptr ? nullptr : a.dfinal_state + state, col, lane);
    } else if (CARRY) {
      dS.load(nullptr, col, lane);
    } else {  // from the segments behind: the last one's is whole
      dS.load(a.carries + (of_segment + a.segments - 1) * D * D, col, lane);
      dS.template cut_all<3>();
      for (int j = a.segments - 2; j > segment; --j)
        advance<D, true>(dS, a.transitions + ((of_segment + j) * 2 + 1) * D * D, a.carries + (of_segment + j) * D * D, col, lane);
    }
    dS.template cut_all<E::kPieces>();
    ColumnTile<E> g;
    g.load(s.of(a.dO, last, a.stride_row), a.stride_row, ~0u, col, lane);
    const Live lives(a, s);
    uint32_t live = lives.bits(lives.fetch(last, lane), last);
    lds_barrier();
    for (int c = last; c >= first; --c) {
      const unsigned char* at = smem + (c & 1) * B::kBytes;
      const float* coef = reinterpret_cast<const float*>(at + B::kCoef);
      const long long chunk = static_cast<long long>(slice) * a.chunks + c;
      if (!CARRY) dS.store(a.dstates + chunk * D * D, col, lane);
      const uint32_t byte = lives.fetch(c > 0 ? c - 1 : 0, lane);
      const Pieces<E::kPieces> up = cut_elements<E>(g.tile(0), g.tile(1));
      const Pieces<3> write = cut<E::kPieces>(g.tile(0) * by_rows(coef + B::kQuery, 0, lane), g.tile(1) * by_rows(coef + B::kQuery, 1, lane));
      if (c > first) g.load(s.of(a.dO, c - 1, a.stride_row), a.stride_row, ~0u, col, lane);
      const Pieces<3> M[2] = {triangle_operand(at + B::kM, 0, lane), triangle_operand(at + B::kM, 1, lane)};
      f32x4_t z[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      add_rows_times<R, D, false>(at + B::kK, dS, z, lane);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) z[tt] *= by_rows(coef + B::kWriteK, tt, lane);
      mul_left(M, up, z);
      const Pieces<3> y = cut<3>(z[0], z[1]);
      const Pieces<3> T[2] = {triangle_operand(at + B::kT, 0, lane), triangle_operand(at + B::kT, 1, lane)};
      z[0] = z[1] = f32x4_t{0, 0, 0, 0};
      mul_left(T, y, z);
      const float whole = coef[B::kWhole];
#pragma unroll
      for (int dt = 0; dt < dS.kTiles; ++dt) dS.s[dt] *= whole;
      add_outer<R, D>(dS, at + B::kQ, write, lane);
      if (!CARRY) {
        store_rows<D>(a.rows_z + chunk * kChunk * D, z, col, lane);
        const __amdgpu_buffer_rsrc_t dV = s.of(a.dV, c, a.stride_row);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          const f32x4_t beta = by_rows(coef + B::kBeta, tt, lane);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = 16 * tt + 4 * (lane >> 4) + r;
            E::store_one(dV, static_cast<uint32_t>(t) * a.stride_row + col * E::kBytes, ((live >> t) & 1u) ? beta[r] * z[tt][r] : 0.0f);
          }
        }
      }
      const Pieces<3> w = cut<E::kPieces>(z[0] * by_rows(coef + B::kAdjoint, 0, lane), z[1] * by_rows(coef + B::kAdjoint, 1, lane));
      add_outer<R, D>(dS, at + B::kK, w, lane);
      dS.template cut_all<E::kPieces>();
      live = lives.bits(byte, c - 1);
      lds_barrier();
    }
    if (CARRY) dS.store(a.carries + (of_segment + segment) * D * D, col, lane);
    else if (segment == 0 && a.dinitial_state != nullptr) dS.store(a.dinitial_state + state, col, lane);
  }
}

// One chunk: a wave has 16 columns (of d_h as the index of q and k) of every result.  Results are computed transposed, so
// a lane has four columns of one token: factors by token are one value, stores are whole pieces of a row.
//
// What bounds it: memory, with the vector units half busy.  128 x 4 x 200 x 64 bf16: 59 us for 250 MB (states on both sides of a
// chunk 32 KB, U and Z 16, rows 24), 4.2 TB/s;  256 x 2 x 200 x 32 fp32: 45 us;  64 x 2 x 197 x 128 fp16: 66 us.  At d = 16 the
// registers for three waves a SIMD do not hold it: 39 of a lane are spilled in fp32, 25 and 23 in 16 bits.
template <class E, int D>
struct GradientLds {
  typedef Rows<D, E::kPieces> R;
  typedef Rows<D, 3> R3;
  static constexpr int kWaves = D / 16;
  static constexpr int kK = 0, kQ = R::kBytes, kG = 2 * R::kBytes, kU = 3 * R::kBytes, kZ = kU + R3::kBytes;
  // the four triangles take the place of U and Z (and, for narrow rows, of what follows), when these have been read
  static constexpr int kTriangles = kU, kRowsEnd = kZ + R3::kBytes, kTrianglesEnd = kTriangles + 4 * kTriangleBytes;
  static constexpr int kSums = kRowsEnd > kTrianglesEnd ? kRowsEnd : kTrianglesEnd;
  // per wave: q^ . dq^, k^ . p, k^ . w, Z . v, r and c by token, <S, dS'>
  static constexpr int kOfWave = 6 * kChunk + 4;
  static constexpr int kPairs = kSums + kWaves * kOfWave * 4;                 // sums of F by token, of its two terms
  static constexpr int kSquares = kPairs + 2 * kChunk * 4;                     // of K's and Q's rows, by block of columns
  static constexpr int kNotes = kSquares + 2 * R::kBlocks * kChunk * 4;        // per wave: what it knows of the tokens
  static constexpr int kBytes = kNotes + kWaves * 5 * kChunk * 4;
};

// What a wave notes of the tokens: sums of decays, beta, 1/r of keys and queries.
struct Tokens {
  float hi[kChunk], lo[kChunk], beta[kChunk], rk[kChunk], rq[kChunk];
  static __device__ __forceinline__ f32x4_t rows(const float* x, int tt, int lane) {  // 16 tt + 4g ... + 3
    return *reinterpret_cast<const f32x4_t*>(x + 16 * tt + 4 * (lane >> 4));
  }
  __device__ __forceinline__ Sum G(int t) const { return Sum{hi[t], lo[t]}; }
};

// sum over i >= t > j of F, t = 0 ... 31, from its tiles (i tile, j tile) (0,0), (1,1), (1,0) as results (row i, column j).
__device__ __forceinline__ void pair_sums(f32x4_t f00, f32x4_t f11, f32x4_t f10, float* to, int lane) {
  const int c = lane & 15, g = lane >> 4;
  // sums over rows from each row on: of the tile's own lane, then of the lane groups behind
  auto suffix = [&](f32x4_t f) {
#pragma unroll
    for (int r = 2; r >= 0; --r) f[r] += f[r + 1];
    const float x1 = __shfl(f[0], (lane + 16) & 63), x2 = __shfl(f[0], (lane + 32) & 63), x3 = __shfl(f[0], (lane + 48) & 63);
    return f + ((g < 3 ? x1 : 0.0f) + (g < 2 ? x2 : 0.0f) + (g < 1 ? x3 : 0.0f));
  };
  const f32x4_t s00 = suffix(f00), s11 = suffix(f11), s10 = suffix(f10);
  const float all10 = __shfl(s10[0], c);
  f32x4_t x, y;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const bool before = c < 4 * g + r;
    const float own = s00[r] + all10, lower = s10[r] + s11[r];
    x[r] = sum_of_row(before ? own : 0.0f);
    y[r] = sum_of_row(before ? lower : s10[r]);
  }
  if (c == 15) {
    *reinterpret_cast<f32x4_t*>(to + 4 * g) = x;
    *reinterpret_cast<f32x4_t*>(to + 16 + 4 * g) = y;
  }
}

// The four triangles (query i, key j; both factors of the unit rows of the operand they meet are in them):
//   0  rows j, columns i:  scale D rk_j (dO U^T)        1  rows i, columns j:  scale D rq_i (dO U^T)
//   2  rows j, columns i: -D rk_j (Z U^T), j < i        3  rows i, columns j: -beta_i D rk_i (Z U^T), j < i
// as tiles (i tile, j tile) (0,0), (1,1), (1,0); of 1 and 3 the sums of F as well.
template <class E, int D, int JOB>
__device__ __forceinline__ void make_triangle(f32x4_t (&m)[3], const unsigned char* at, const Tokens& n, float scale, float* pairs,
                                              int lane) {
  typedef GradientLds<E, D> L;
  typedef typename L::R R;
  typedef typename L::R3 R3;
  constexpr bool kByI = (JOB & 1) != 0, kOuter = JOB < 2;
  const int c = lane & 15, g = lane >> 4;
  const f32x4_t zero = {0, 0, 0, 0};
  m[0] = m[1] = m[2] = zero;
  f32x4_t d00 = zero, d11 = zero, d10 = zero;
#pragma unroll
  for (int kb = 0; kb < R::kBlocks; ++kb) {
    const Pieces<3> u0 = R3::row_operand(at + L::kU, 0, kb, lane), u1 = R3::row_operand(at + L::kU, 1, kb, lane);
    auto products = [&](const auto& x0, const auto& x1) {
      m[0] = kByI ? mul(x0, u0, m[0]) : mul(u0, x0, m[0]);
      m[1] = kByI ? mul(x1, u1, m[1]) : mul(u1, x1, m[1]);
      m[2] = kByI ? mul(x1, u0, m[2]) : mul(u0, x1, m[2]);
    };
    if constexpr (kOuter) products(R::row_operand(at + L::kG, 0, kb, lane), R::row_operand(at + L::kG, 1, kb, lane));
    else products(R3::row_operand(at + L::kZ, 0, kb, lane), R3::row_operand(at + L::kZ, 1, kb, lane));
    if constexpr (kByI) {
      const auto x0 = R::row_operand(at + (kOuter ? L::kQ : L::kK), 0, kb, lane), x1 = R::row_operand(at + (kOuter ? L::kQ : L::kK), 1, kb, lane);
      const auto k0 = R::row_operand(at + L::kK, 0, kb, lane), k1 = R::row_operand(at + L::kK, 1, kb, lane);
      d00 = mul(x0, k0, d00);
      d11 = mul(x1, k1, d11);
      d10 = mul(x1, k0, d10);
    }
  }
  const float* factor = JOB == 1 ? n.rq : n.rk;
  f32x4_t f0 = Tokens::rows(factor, 0, lane), f1 = Tokens::rows(factor, 1, lane);
  if (kOuter) {
    f0 *= scale;
    f1 *= scale;
  } else {
    f0 *= kByI ? -Tokens::rows(n.beta, 0, lane) : f32x4_t{-1, -1, -1, -1};
    f1 *= kByI ? -Tokens::rows(n.beta, 1, lane) : f32x4_t{-1, -1, -1, -1};
  }
  const f32x4_t hi0 = Tokens::rows(n.hi, 0, lane), hi1 = Tokens::rows(n.hi, 1, lane), lo0 = Tokens::rows(n.lo, 0, lane),
                lo1 = Tokens::rows(n.lo, 1, lane);
  const Sum c0 = n.G(c), c1 = n.G(16 + c);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int o = 4 * g + r;
    const Sum o0{hi0[r], lo0[r]}, o1{hi1[r], lo1[r]};
    const float x0 = m[0][r] * f0[r] * (kByI ? pow2(o0, c0) : pow2(c0, o0));
    const float x1 = m[1][r] * f1[r] * (kByI ? pow2(o1, c1) : pow2(c1, o1));
    const bool in = kByI ? (kOuter ? o >= c : o > c) : (kOuter ? o <= c : o < c);
    m[0][r] = in ? x0 : 0.0f;
    m[1][r] = in ? x1 : 0.0f;
    m[2][r] *= kByI ? f1[r] * pow2(o1, c0) : f0[r] * pow2(c1, o0);
  }
  if constexpr (kByI) {
    const float r0 = n.rk[c], r1 = n.rk[16 + c];
    d00 *= m[0] * r0;
    d11 *= m[1] * r1;
    d10 *= m[2] * r0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool in = 4 * g + r > c;
      d00[r] = in ? d00[r] : 0.0f;
      d11[r] = in ? d11[r] : 0.0f;
    }
    pair_sums(d00, d11, d10, pairs + (JOB >> 1) * kChunk, lane);
  }
}
template <int JOB, int OTHER>
__device__ __forceinline__ void put_tiles(unsigned char* at, const f32x4_t (&m)[3], int lane) {
  const f32x4_t zero = {0, 0, 0, 0};
  put_triangle<OTHER>(at + JOB * kTriangleBytes, 0, lane, m[0], (JOB & 1) ? m[2] : zero);
  put_triangle<OTHER>(at + JOB * kTriangleBytes, 1, lane, (JOB & 1) ? zero : m[2], m[1]);
}

template <class E, int D>
__global__ __launch_bounds__(64 * (D / 16), D == 128 ? 2 : 3) void chunk_gradient_kernel(Args a) {
  typedef GradientLds<E, D> L;
  typedef typename L::R R;
  typedef typename L::R3 R3;
  constexpr int kWaves = L::kWaves, kBlocks = R::kBlocks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, gr = lane >> 4;
  const uint32_t chunk = blockIdx.x;
  const int slice = chunk / a.chunks, c = chunk - slice * a.chunks;
  const Slice s(a, slice, D * E::kBytes);
  const Live lives(a, s);
  const uint32_t live = lives.bits(lives.fetch(c, lane), c), there = existing(a.N, c);
  const __amdgpu_buffer_rsrc_t Q = s.of(a.Q, c, a.stride_row), K = s.of(a.K, c, a.stride_row), V = s.of(a.V, c, a.stride_row);
  Tokens& n = *reinterpret_cast<Tokens*>(smem + L::kNotes + wave * sizeof(Tokens));

  // K, Q, dO, U, Z: a wave brings 16 rows of 32 columns of each (d = 16: all of them), everything at once
  constexpr int kUnits = kWaves == 1 ? 2 : 1;
  typename E::Raw raw[kUnits][3];
  F32::Raw wide[kUnits][2];
  const int kb0 = kWaves == 1 ? 0 : wave >> 1;
  const uint32_t state_rows = kChunk * D * 4;
  const __amdgpu_buffer_rsrc_t rows_u = buffer(a.rows_u + static_cast<long long>(chunk) * kChunk * D, state_rows);
  const __amdgpu_buffer_rsrc_t rows_z = buffer(a.rows_z + static_cast<long long>(chunk) * kChunk * D, state_rows);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int row = 16 * (kWaves == 1 ? u : wave & 1) + c16, col = 32 * kb0 + 8 * gr;
    const bool inside = D >= 32 || col < D;
    const uint32_t off = inside ? static_cast<uint32_t>(row) * a.stride_row + col * E::kBytes : kNowhere;
    raw[u][0] = E::load(K, offset_if(live, row, off));
    raw[u][1] = E::load(Q, off);
    raw[u][2] = E::load(s.of(a.dO, c, a.stride_row), off);
    wide[u][0] = F32::load(rows_u, inside ? (row * D + col) * 4 : kNowhere);
    wide[u][1] = F32::load(rows_z, inside ? (row * D + col) * 4 : kNowhere);
  }
  const bool on = (live >> (lane & 31)) & 1u;
  const float g = __uint_as_float(fetch_gate(a, s.of_gate(a, a.g), c, live, lane)),
              beta = __uint_as_float(fetch_gate(a, s.of_gate(a, a.beta), c, live, lane));
  StateRows<D> before, after;
  before.load(a.states + static_cast<long long>(chunk) * D * D, wave, lane);
  after.load(a.dstates + static_cast<long long>(chunk) * D * D, wave, lane);
  // a lane's four columns of its two tokens
  f32x4_t q[2], k[2], zv[2];
  uint32_t off[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    off[tt] = static_cast<uint32_t>(t) * a.stride_row + (16 * wave + 4 * gr) * E::kBytes;
    q[tt] = E::load_four(Q, off[tt]);
    k[tt] = E::load_four(K, offset_if(live, t, off[tt]));
    zv[tt] = E::load_four(V, offset_if(live, t, off[tt])) * F32::load_four(rows_z, (t * D + 16 * wave + 4 * gr) * 4);
  }
  float* squares = reinterpret_cast<float*>(smem + L::kSquares);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int row = 16 * (kWaves == 1 ? u : wave & 1) + c16;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x[8], ss = 0.0f;
      E::unpack(raw[u][i], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
      ss = over_groups(ss);
      squares[(i * kBlocks + kb0) * kChunk + row] = ss;  // (the four lanes of a row: the same)
    }
    R::put(smem + L::kK, row, kb0, gr, E::pieces(raw[u][0]));
    R::put(smem + L::kQ, row, kb0, gr, E::pieces(raw[u][1]));
    R::put(smem + L::kG, row, kb0, gr, E::pieces(raw[u][2]));
    R3::put(smem + L::kU, row, kb0, gr, F32::pieces(wide[u][0]));
    R3::put(smem + L::kZ, row, kb0, gr, F32::pieces(wide[u][1]));
  }
  const Sum G = scan_decays(g, lane), G_end = last_of_scan(G);
  lds_barrier();
  {
    const int t = lane & 31;
    float kk = a.eps, qq = a.eps;
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
      kk += squares[kb * kChunk + t];
      qq += squares[(kBlocks + kb) * kChunk + t];
    }
    n.hi[t] = G.hi;
    n.lo[t] = G.lo;
    n.beta[t] = beta;
    n.rk[t] = on ? __builtin_amdgcn_rsqf(kk) : 0.0f;  // (rows that were not loaded: 0 whatever eps is)
    n.rq[t] = ((there >> t) & 1u) ? __builtin_amdgcn_rsqf(qq) : 0.0f;
  }
  wave_fence();

  float* pairs = reinterpret_cast<float*>(smem + L::kPairs);
  f32x4_t m[kWaves >= 4 ? 1 : 4 / kWaves][3];
  if constexpr (kWaves >= 4) {
    if (wave == 0) make_triangle<E, D, 0>(m[0], smem, n, a.scale, pairs, lane);
    else if (wave == 1) make_triangle<E, D, 1>(m[0], smem, n, a.scale, pairs, lane);
    else if (wave == 2) make_triangle<E, D, 2>(m[0], smem, n, a.scale, pairs, lane);
    else if (wave == 3) make_triangle<E, D, 3>(m[0], smem, n, a.scale, pairs, lane);
  } else if constexpr (kWaves == 2) {
    if (wave == 0) {
      make_triangle<E, D, 0>(m[0], smem, n, a.scale, pairs, lane);
      make_triangle<E, D, 3>(m[1], smem, n, a.scale, pairs, lane);
    } else {
      make_triangle<E, D, 1>(m[0], smem, n, a.scale, pairs, lane);
      make_triangle<E, D, 2>(m[1], smem, n, a.scale, pairs, lane);
    }
  } else {
    make_triangle<E, D, 0>(m[0], smem, n, a.scale, pairs, lane);
    make_triangle<E, D, 1>(m[1], smem, n, a.scale, pairs, lane);
    make_triangle<E, D, 2>(m[2], smem, n, a.scale, pairs, lane);
    make_triangle<E, D, 3>(m[3], smem, n, a.scale, pairs, lane);
  }

  // what the states give, tokens in columns
  f32x4_t dq[2], p[2], w[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) dq[tt] = p[tt] = w[tt] = f32x4_t{0, 0, 0, 0};
  float inner = 0.0f;  // <S, dS'> over the wave's columns
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb) {
    const Pieces<3> S = cut<3>(before.lo[kb], before.hi[kb]), dS = cut<3>(after.lo[kb], after.hi[kb]);
    const Pieces<E::kPieces> up[2] = {R::row_operand(smem + L::kG, 0, kb, lane), R::row_operand(smem + L::kG, 1, kb, lane)};
    mul_right(S, up, dq);
    const Pieces<3> z[2] = {R3::row_operand(smem + L::kZ, 0, kb, lane), R3::row_operand(smem + L::kZ, 1, kb, lane)};
    mul_right(S, z, p);
    const Pieces<3> u[2] = {R3::row_operand(smem + L::kU, 0, kb, lane), R3::row_operand(smem + L::kU, 1, kb, lane)};
    mul_right(dS, u, w);
#pragma unroll
    for (int r = 0; r < 4; ++r) inner += before.lo[kb][r] * after.lo[kb][r] + before.hi[kb][r] * after.hi[kb][r];
  }
  lds_barrier();  // U and Z have been read
  unsigned char* triangles = smem + L::kTriangles;
  if constexpr (kWaves >= 4) {
    if (wave == 0) put_tiles<0, E::kPieces>(triangles, m[0], lane);
    else if (wave == 1) put_tiles<1, E::kPieces>(triangles, m[0], lane);
    else if (wave == 2) put_tiles<2, E::kPieces>(triangles, m[0], lane);
    else if (wave == 3) put_tiles<3, E::kPieces>(triangles, m[0], lane);
  } else if constexpr (kWaves == 2) {
    if (wave == 0) {
      put_tiles<0, E::kPieces>(triangles, m[0], lane);
      put_tiles<3, E::kPieces>(triangles, m[1], lane);
    } else {
      put_tiles<1, E::kPieces>(triangles, m[0], lane);
      put_tiles<2, E::kPieces>(triangles, m[1], lane);
    }
  } else {
    put_tiles<0, E::kPieces>(triangles, m[0], lane);
    put_tiles<1, E::kPieces>(triangles, m[1], lane);
    put_tiles<2, E::kPieces>(triangles, m[2], lane);
    put_tiles<3, E::kPieces>(triangles, m[3], lane);
  }
  inner *= pow2(G_end);
  float read[2], write[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    const Sum Gt = n.G(t);
    const float eG = pow2(Gt);
    q[tt] *= n.rq[t];
    k[tt] *= n.rk[t];
    dq[tt] *= a.scale * eG;
    p[tt] *= -eG;
    w[tt] *= pow2(G_end, Gt);
    float x = 0.0f, y = 0.0f, z = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x = fmaf(q[tt][r], dq[tt][r], x);
      y = fmaf(k[tt][r], p[tt][r], y);
      z = fmaf(k[tt][r], w[tt][r], z);
    }
    read[tt] = fmaf(n.beta[t], y, x);
    write[tt] = z;
  }
  lds_barrier();
  {
    const Pieces<E::kPieces> kc = R::column_operand(smem + L::kK, wave, lane), qc = R::column_operand(smem + L::kQ, wave, lane);
    auto add = [&](const Pieces<E::kPieces>& x, int triangle, f32x4_t (&c)[2]) {
      const unsigned char* at = triangles + triangle * kTriangleBytes;
      const Pieces<3> t[2] = {triangle_operand(at, 0, lane), triangle_operand(at, 1, lane)};
      mul_right(x, t, c);
    };
    add(kc, 0, dq);
    add(kc, 2, p);
    add(qc, 1, w);
    add(kc, 3, w);
  }
  // products of a row with its gradients, over all columns
  float* sums = reinterpret_cast<float*>(smem + L::kSums);
  float* own = sums + wave * L::kOfWave;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    float qd = 0.0f, kp = 0.0f, kw = 0.0f, v = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      qd = fmaf(q[tt][r], dq[tt][r], qd);
      kp = fmaf(k[tt][r], p[tt][r], kp);
      kw = fmaf(k[tt][r], w[tt][r], kw);
      v += zv[tt][r];
    }
    qd = over_groups(qd);
    kp = over_groups(kp);
    kw = over_groups(kw);
    v = over_groups(v);
    const float reads = over_groups(read[tt]), writes = over_groups(write[tt]);
    // lane group gr keeps the gr-th of them
    own[gr * kChunk + t] = (gr & 2) ? ((gr & 1) ? v : kw) : ((gr & 1) ? kp : qd);
    if (gr < 2) own[(4 + gr) * kChunk + t] = gr == 0 ? reads : writes;
  }
  inner = over_groups(sum_of_row(inner));
  if (lane == 15) own[6 * kChunk] = inner;
  lds_barrier();
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    const float b = n.beta[t];
    float qd = 0.0f, kp = 0.0f, kw = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      qd += sums[i * L::kOfWave + t];
      kp += sums[i * L::kOfWave + kChunk + t];
      kw += sums[i * L::kOfWave + 2 * kChunk + t];
    }
    const float kd = fmaf(b, kp, kw), rq = n.rq[t], rk = n.rk[t];
    f32x4_t x, y;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[r] = (dq[tt][r] - q[tt][r] * qd) * rq;
      y[r] = (fmaf(b, p[tt][r], w[tt][r]) - k[tt][r] * kd) * rk;
      y[r] = ((live >> t) & 1u) ? y[r] : 0.0f;
    }
    E::store_four(s.of(a.dQ, c, a.stride_row), off[tt], x);
    E::store_four(s.of(a.dK, c, a.stride_row), off[tt], y);
  }
  if (wave == kWaves - 1) {
    const int t = lane & 31;
    float kp = 0.0f, v = 0.0f, reads = 0.0f, writes = 0.0f, end = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float* of = sums + i * L::kOfWave;
      kp += of[kChunk + t];
      v += of[3 * kChunk + t];
      reads += of[4 * kChunk + t];
      writes += t > 0 ? of[5 * kChunk + t - 1] : 0.0f;  // of the tokens before
      end += of[6 * kChunk];
    }
    const float x = pairs[t] + pairs[kChunk + t] + sums_from(reads, lane) + sums_up_to(writes, lane) + end;
    const long long gate = s.gates + (static_cast<long long>(kChunk) * c + t) * a.gate_row;
    if (lane < 32 && ((there >> t) & 1u)) {
      a.dg[gate] = on ? x : 0.0f;
      a.dbeta[gate] = on ? v + kp : 0.0f;
    }
  }
}

template <class E, int D, bool CARRY>
hipError_t launch_walk(const Args& a, int slices, hipStream_t stream) {
  constexpr int kLds = kWalkLds<E, D>;
  const auto kernel = chunk_adjoint_kernel<E, D, CARRY>;
  if (hipError_t err = grant_dynamic_lds(reinterpret_cast<const void*>(kernel), kLds); err != hipSuccess) return err;
  const int walked = CARRY ? a.segments - 1 : a.segments;
  kernel<<<dim3(slices * walked * (D / 16 / kConsumers<D>)), dim3(64 * (kConsumers<D> + 2)), kLds, stream>>>(a);
  return hipGetLastError();
}

template <class E, int D>
hipError_t launch(const Args& a, int slices, hipStream_t stream) {
  if (a.segments > 1)
    if (hipError_t err = launch_walk<E, D, true>(a, slices, stream); err != hipSuccess) return err;
  if (hipError_t err = launch_walk<E, D, false>(a, slices, stream); err != hipSuccess) return err;
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
