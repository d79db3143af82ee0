// Forward of the gated delta rule (cotten_delta_core.h has the formulas): a recurrence for a few tokens, and chunks of 32
// tokens on the matrix cores for more.
#include "cotten_delta_chunk.h"
#include "cotten_delta_launch.h"
#include "cotten_launch.h"

namespace cotten {
namespace delta {
namespace {

extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

// ---- token by token -----------------------------------------------------------------------------------------------
//
// A wave carries up to 32 columns of a state in registers (columns do not meet: u of a column needs that column only),
// eight lanes to a row of 128 bytes, the rows dealt to the lane groups.  k^ . S and q^ . S are sums over the groups by
// lane permutes; no LDS, no barrier.  One token is bound by the state, read and written once: 1024 x 4 states of 64 x 64 in
// 21.4 us, 6.3 TB/s (the memory-side cache helps); 4 x 2 states of 32 x 32 in 3.8 us, a launch and three trips to memory.
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
  const __amdgpu_buffer_rsrc_t Q = s.of(a.Q), K = s.of(a.K), V = s.of(a.V), O = s.of(a.O);

  f32x4_t S[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    S[r] = a.initial_state == nullptr
               ? f32x4_t{0, 0, 0, 0}
               : *reinterpret_cast<const f32x4_t*>(a.initial_state + (static_cast<long long>(slice) * D + group + r * kGroups) * D + col);
  for (int t = 0; t < a.N; ++t) {
    const bool live = s.mask == nullptr || s.mask[t] != 0;
    const uint32_t row = static_cast<uint32_t>(t) * a.stride_row;
    const long long gate = s.gates + static_cast<long long>(t) * a.gate_row;
    const float decay = live ? expf(a.g[gate]) : 1.0f, beta = live ? a.beta[gate] : 0.0f;
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
    f32x4_t p = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      S[r] *= decay;
#pragma unroll
      for (int c = 0; c < 4; ++c) p[c] = fmaf(k[r], S[r][c], p[c]);
    }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
      kk += __shfl_xor(kk, m);
      qq += __shfl_xor(qq, m);
#pragma unroll
      for (int c = 0; c < 4; ++c) p[c] += __shfl_xor(p[c], m);
    }
    const float rk = __builtin_amdgcn_rsqf(kk + a.eps), rq = a.scale * __builtin_amdgcn_rsqf(qq + a.eps);
    f32x4_t u, o = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < 4; ++c) u[c] = live ? beta * (v[c] - rk * p[c]) * rk : 0.0f;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        S[r][c] = fmaf(k[r], u[c], S[r][c]);
        o[c] = fmaf(q[r], S[r][c], o[c]);
      }
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += __shfl_xor(o[c], m);
    if (group == 0) E::store_four(O, row + col * E::kBytes, o * rq);
  }
  if (a.final_state != nullptr) {
#pragma unroll
    for (int r = 0; r < kRows; ++r)
      *reinterpret_cast<f32x4_t*>(a.final_state + (static_cast<long long>(slice) * D + group + r * kGroups) * D + col) = S[r];
  }
}

// ---- chunks ---------------------------------------------------------------------------------------------------------
//
// A workgroup walks the chunks of a slice: wave 0 makes the keys' side of a chunk, wave 1 the queries', the others carry 16
// columns of the state each, a chunk behind.  Everything a consumer passes on to itself (K^ S -> U -> O, S) stays in the
// registers it came out in; LDS only carries what the producers made.
//
// What bounds it: the keys' producer, whose chunk (rows, products, norms, decays, the solve, T) is one chain of 440 vector
// instructions and the trips to LDS between them.  A chunk of d = 64 in bf16 takes 2160 vector and 270 matrix instructions
// over the six waves, 900 of them to cut results into pieces: 1.8 us for a workgroup alone on a compute unit (producers without
// consumers 1.5, consumers without producers 1.45) and 1.6 for each of two that share one (1.6 and 1.1: the consumers hide).
// Times of calls in a loop: 128 x 4 x 200 x 64 bf16 25.2 us, 4.2 TB/s of its tensors;  256 x 2 x 200 x 32 fp32
// 21.0;  64 x 2 x 197 x 128 fp16 30.2;  16 x 4 x 4096 x 64 bf16 in four segments 129, half of it for the segments' R and M (nine waves
// a workgroup).  Timed apart: 256 x 2 x 200 x 16 bf16 16.8, fp32 22.3;  128 x 2 x 200 x 128 bf16 39.4, fp32 110 (80 registers of a
// lane are spilled there).
template <int D>
constexpr int kConsumers = D / 16 < 4 ? D / 16 : 4;  // of a workgroup; d = 128 takes two (of ten waves, none would have the registers)

// What a walk is for: O; O and what a backward needs; the latter alone; a segment's R and M (see segments_of).
enum Walk { kOutput, kTraining, kStates, kTransition };

template <int D, Walk WALK>
constexpr int kProducers = WALK == kOutput || WALK == kTraining ? 2 : 1;
template <int D, Walk WALK>
constexpr int kWaves = kProducers<D, WALK> + kConsumers<D> * (WALK == kTransition ? 2 : 1);

template <class E, int D, Walk WALK>
constexpr int kLds = 2 * ChunkBuffer<E, D, kProducers<D, WALK> == 2>::kBytes + sizeof(Scratch) + sizeof(Notes);

template <class E, int D, Walk WALK>
__global__ __launch_bounds__(64 * (kWaves<D, WALK>), waves_per_simd(kWaves<D, WALK>, kLds<E, D, WALK>)) void chunk_fwd_kernel(Args a) {
  constexpr bool kOut = WALK == kOutput || WALK == kTraining;
  typedef ChunkBuffer<E, D, kOut> B;
  typedef typename B::R R;
  constexpr bool kKept = WALK == kTraining || WALK == kStates;
  constexpr int kGroups = D / 16 / kConsumers<D>;
  const int lane = threadIdx.x & 63, wave = role_of_wave<(kWaves<D, WALK>)>();
  const int unit = blockIdx.x / kGroups, group = blockIdx.x % kGroups;
  const int walked = WALK == kTransition ? a.segments - 1 : a.segments;
  const int slice = unit / walked, segment = unit - slice * walked;
  const Slice s(a, slice, D * E::kBytes);
  Scratch* scratch = reinterpret_cast<Scratch*>(smem + 2 * B::kBytes);
  Notes* notes = reinterpret_cast<Notes*>(scratch + 1);
  const int first = segment * a.segment_chunks;
  const int end = first + a.segment_chunks < a.chunks ? first + a.segment_chunks : a.chunks;

  if (wave == 0) {
    KeyProducer<E, D, false, kOut> producer(a, s);
    producer.begin(first, first + 1, lane);
    for (int c = first; c <= end; ++c) {
      if (c < end) producer.make(c + 1, c + 2, smem + (c & 1) * B::kBytes, scratch, lane);
      lds_barrier();
    }
  } else if (kOut && wave == 1) {
    QueryProducer<E, D, false> producer(a, s);
    producer.begin(first, first + 1, lane);
    for (int c = first; c <= end; ++c) {
      if (c < end) producer.make(c + 1, c + 2, smem + (c & 1) * B::kBytes, notes, lane);
      lds_barrier();
    }
  } else {
    const int consumer = wave - kProducers<D, WALK>;
    const bool is_m = WALK == kTransition && consumer >= kConsumers<D>;
    const int tile = group * kConsumers<D> + consumer % kConsumers<D>, col = 16 * tile + (lane & 15);
    const long long of_segment = static_cast<long long>(slice) * a.segments;
    const float* initial = a.initial_state == nullptr ? nullptr : a.initial_state + static_cast<long long>(slice) * D * D;
    StateColumns<D> S;
    if (is_m && segment == 0) {
      // nobody needs the first segment's M (its R has the initial state in it): a copy of the initial state takes the place.
      // The next launch starts from the copy, as final_state may be initial_state and another workgroup writes it.
      S.load(initial, col, lane);
      S.store(a.transitions + (of_segment * 2 + 1) * D * D, col, lane);
      for (int c = first; c <= end; ++c) lds_barrier();
      return;
    }
    if (is_m) {
      S.unit(col, lane);
    } else if (segment == 0) {
      S.load(WALK != kTransition && a.segments > 1 ? a.transitions + (of_segment * 2 + 1) * D * D : initial, col, lane);
    } else if (WALK == kTransition) {
      S.load(nullptr, col, lane);
    } else {  // from the segments before: the first one's R has the initial state in it
      S.load(a.transitions + of_segment * 2 * D * D, col, lane);
      S.template cut_all<3>();
      for (int j = 1; j < segment; ++j) {
        const float* R = a.transitions + (of_segment + j) * 2 * D * D;
        advance<D, false>(S, R + D * D, R, col, lane);
      }
    }
    S.template cut_all<E::kPieces>();
    ColumnTile<E> v;
    const Live lives(a, s);
    const uint32_t with_v = is_m ? 0u : ~0u;
    v.load(s.of(a.V, first, a.stride_row), a.stride_row, with_v & lives.bits(lives.fetch(first, lane), first), col, lane);
    uint32_t byte = lives.fetch(first + 1, lane);
    lds_barrier();
    for (int c = first; c < end; ++c) {
      const unsigned char* at = smem + (c & 1) * B::kBytes;
      const float* coef = reinterpret_cast<const float*>(at + B::kCoef);
      const long long chunk = static_cast<long long>(slice) * a.chunks + c;
      if (kKept) S.store(a.states + chunk * D * D, col, lane);
      // beta (V - e^G K^ S)
      f32x4_t u[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      add_rows_times<R, D, false>(at + B::kK, S, u, lane);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
        u[tt] = by_rows(coef + B::kBeta, tt, lane) * (v.tile(tt) - by_rows(coef + B::kReadK, tt, lane) * u[tt]);
      if (c + 1 < end) {
        v.load(s.of(a.V, c + 1, a.stride_row), a.stride_row, with_v & lives.bits(byte, c + 1), col, lane);
        byte = lives.fetch(c + 2, lane);
      }
      const Pieces<3> y = cut<3>(u[0], u[1]);
      const Pieces<3> T[2] = {triangle_operand(at + B::kT, 0, lane), triangle_operand(at + B::kT, 1, lane)};
      u[0] = u[1] = f32x4_t{0, 0, 0, 0};
      mul_left(T, y, u);
      // O^T: a lane has four columns of a token; the state's part of it while U comes
      f32x4_t o[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      if (kOut) add_rows_times<R, D, true>(at + B::kQ, S, o, lane);
      if (kKept) store_rows<D>(a.rows_u + chunk * kChunk * D, u, col, lane);
      // S' = e^(G_C) S + K^^T (e^(G_C - G) U)
      const float whole = coef[B::kWhole];
      const Pieces<3> w = cut<E::kPieces>(u[0] * by_rows(coef + B::kWriteK, 0, lane), u[1] * by_rows(coef + B::kWriteK, 1, lane));
#pragma unroll
      for (int dt = 0; dt < S.kTiles; ++dt) S.s[dt] *= whole;
      add_outer<R, D>(S, at + B::kK, w, lane);
      if (kOut) {
        const __amdgpu_buffer_rsrc_t O = s.of(a.O, c, a.stride_row);
        const Pieces<3> up = cut<3>(u[0], u[1]);
        const Pieces<3> M[2] = {triangle_operand(at + B::kM, 0, lane), triangle_operand(at + B::kM, 1, lane)};
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) o[tt] *= coef[B::kQuery + 16 * tt + (lane & 15)];
        mul_right(up, M, o);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
          E::store_four(O, static_cast<uint32_t>(16 * tt + (lane & 15)) * a.stride_row + (16 * tile + 4 * (lane >> 4)) * E::kBytes, o[tt]);
      }
      S.template cut_all<E::kPieces>();
      lds_barrier();
    }
    if (WALK == kTransition) S.store(a.transitions + ((of_segment + segment) * 2 + (is_m ? 1 : 0)) * D * D, col, lane);
    else if (end == a.chunks && a.final_state != nullptr) S.store(a.final_state + static_cast<long long>(slice) * D * D, col, lane);
  }
}

// Up to how many tokens a call runs as a recurrence.  Every token takes it a microsecond or two more; a chunk takes what it
// takes, which grows with the workgroups that share a compute unit, more where operands are three pieces.  Measured (us,
// recurrence / chunk):  256 slices of d = 64, bf16: 6 tokens 9.8 / 9.5, 8 tokens 11.2 / 9.5;  1024: 8 tokens 15.1 / 15.6, 10
// tokens 18.3 / 15.7;  2048: 10 tokens about 26 / 28, fp32: 16 tokens 38 / 47, 24 tokens 52 / 47;  1024 of d = 128, bf16: 10
// tokens 40 / 42, 12 tokens 44 / 43, fp16: 12 tokens 51 / 55, 16 tokens 63 / 56.
template <class E, int D>
int most_steps(int slices) {
  const long long workgroups = static_cast<long long>(slices) * (D / 16 / kConsumers<D>);
  return workgroups <= 512 ? 6 : workgroups <= 1024 ? 8 : E::kPieces == 3 ? 16 : 10;
}

template <class E, int D, Walk WALK>
hipError_t launch_chunks(const Args& a, int slices, hipStream_t stream) {
  constexpr int lds = kLds<E, D, WALK>;
  const auto kernel = chunk_fwd_kernel<E, D, WALK>;
  if (hipError_t err = grant_dynamic_lds(reinterpret_cast<const void*>(kernel), lds); err != hipSuccess) return err;
  const int walked = WALK == kTransition ? a.segments - 1 : a.segments;
  kernel<<<dim3(slices * walked * (D / 16 / kConsumers<D>)), dim3(64 * kWaves<D, WALK>), lds, stream>>>(a);
  return hipGetLastError();
}

template <class E, int D>
hipError_t launch(const Args& a, int slices, hipStream_t stream) {
  const bool out = a.O != nullptr, kept = a.states != nullptr;
  if (out && !kept && a.N <= most_steps<E, D>(slices)) {
    constexpr int kParts = D < 32 ? 1 : D / 32;
    const long long waves = static_cast<long long>(slices) * kParts;
    const int per = waves >= 4096 ? 4 : 1;  // few waves go to a compute unit each (512 x 2 x 128 fp32: 20.3 us in fours, 21.0 alone)
    step_kernel<E, D><<<dim3(static_cast<uint32_t>((waves + per - 1) / per)), dim3(64 * per), 0, stream>>>(a, slices);
    return hipGetLastError();
  }
  if (a.segments > 1)
    if (hipError_t err = launch_chunks<E, D, kTransition>(a, slices, stream); err != hipSuccess) return err;
  return !out   ? launch_chunks<E, D, kStates>(a, slices, stream)
         : kept ? launch_chunks<E, D, kTraining>(a, slices, stream)
                : launch_chunks<E, D, kOutput>(a, slices, stream);
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

Segments segments_of(long long slices, int chunks, int D, int dtype) {
  // About one workgroup for each of the 256 compute units (two take as long as one after the other): 16 x 4 x 4096 x 64
  // bf16, forward / backward: whole 242 / 378 us, in 4 segments 135 / 287 (129 / 282 by now), in 8 146 / 303; 16 x 4 x 1024: whole 64 / 98, 4
  // segments 43 / 74.  Not more segments than make up for the steps M S + R over them (one takes about as long as half a
  // chunk in each of the two launches).  With two the first launch takes what the second saves: 32 x 4 x 2048 whole 123 /
  // 261 us, in 2 segments 120 / 273;  20 x 4 x 2048 whole 123 / 206, in 3 93 / 183.
  //
  // Few chunks do not make up for the second launch and the steps, which take four times as long at twice the width.  In
  // segments / whole, us: d = 16 and 32, seven chunks 12 ... 14 % longer for bf16 and 6 ... 11 % for fp32, eight (16 x 4 x 256 x
  // 32 bf16) forward 13.9 / 15.2, backward 22.6 / 25.2;  d = 64 bf16, 16 x 4 of eight chunks 21.5 / 18.2 and 32.3 / 34.9, of nine
  // 20.6 / 19.9 and 37.9 / 39.6, of 12 25.2 / 25.2 and 39.9 / 45.1, fp32 of nine 26.1 / 27.3 and 49.9 / 52.1;  d = 128 bf16, 4 x 4
  // of 12 41 / 31 and 53 / 54, of 17 45.5 / 42.5 and 77 / 78, with the states kept 47.5 / 47.9, of 24 60 / 58.5, 63 / 65.5 and
  // 84 / 96, fp16 of 17 55 / 66 and 90 / 104, fp32 of nine 49 / 60 and 86 / 91.
  constexpr int kWorkgroups = 256, kFewest = 3;
  const long long groups = slices * (D > 64 ? D / 64 : 1);
  long long count = kWorkgroups / groups < chunks ? kWorkgroups / groups : chunks;
  while (count * count > 2ll * chunks) --count;
  const int fewest_chunks = D <= 32 ? 8 : D == 64 || dtype == 0 ? 9 : 17;
  if (count < kFewest || chunks < fewest_chunks) return Segments{1, chunks};
  const int each = static_cast<int>((chunks + count - 1) / count);
  return Segments{(chunks + each - 1) / each, each};
}

hipError_t launch_forward(const Args& a, int dtype, int D, int slices, hipStream_t stream) {
  return dtype == 0 ? launch_dim<F32>(a, D, slices, stream)
         : dtype == 1 ? launch_dim<Bf16>(a, D, slices, stream)
                      : launch_dim<F16>(a, D, slices, stream);
}

}  // namespace delta
}  // namespace cotten
