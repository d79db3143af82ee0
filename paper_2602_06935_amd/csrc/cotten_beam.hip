// A step of a beam search: the best K of the K * V continuations of every sequence's K beams, and the reordering of what
// belongs to the beams.
//
//     total[k, v] = score[k] + logit[k, v] - log sum_v' exp(logit[k, v'])        a beam that ended: score[k] at the pad
//                                                                                 item, -inf elsewhere
//
// The best, the lower k * V + v of equal ones first.  Within a beam the order of the totals is that of the logits, so a row of
// logits is read once, in parts: a wave keeps the K best of its part (value and item) and the sum of the exponentials, and
// one workgroup a sequence joins what the parts of its K rows hold, with totals in 64 bits.  The exponentials are fp32, which leaves
// the logarithm of a row's sum right to 2e-6 at worst (how_near) and some 1e-8 as a rule; where candidates of two beams come nearer than
// that, the sums of these rows are made again in 64 bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/cotten_attn.h"

namespace cotten {
namespace beam {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kMostBeams = 32;

// A logit and its item as one number: greater is ahead.  The float's bits are turned so that they count up with the value (-0
// counts as 0, NaN as -inf), the item's are inverted.
__device__ __forceinline__ uint32_t in_order(float x) {
  x = x != x ? -__builtin_inff() : x + 0.0f;
  const uint32_t b = __float_as_uint(x);
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_order(uint32_t u) { return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t item) { return (static_cast<uint64_t>(in_order(x)) << 32) | ~item; }

// The value of lane ^ M, without a trip through LDS: quads, rows of 16 and halves of a wave have moves of their own.
template <int CTRL>
__device__ __forceinline__ uint32_t move(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xF, 0xF, true));
}
template <int M>
__device__ __forceinline__ uint32_t of_xor(uint32_t x, int lane) {
  if constexpr (M == 1) return move<0xB1>(x);               // quad_perm 1,0,3,2
  else if constexpr (M == 2) return move<0x4E>(x);          // quad_perm 2,3,0,1
  else if constexpr (M == 4) return move<0x1B>(move<0x141>(x));  // the eight reversed, then the fours
  else if constexpr (M == 8) return move<0x128>(x);         // row_ror 8
  else if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return (lane & 16) ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (lane & 32) ? r[0] : r[1];
  }
}
template <int M>
__device__ __forceinline__ uint64_t of_xor(uint64_t x, int lane) {
  return (static_cast<uint64_t>(of_xor<M>(static_cast<uint32_t>(x >> 32), lane)) << 32) | of_xor<M>(static_cast<uint32_t>(x), lane);
}
__device__ __forceinline__ uint64_t shuffle(uint64_t x, int lane) {
  return (static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(x >> 32), lane))) << 32) |
         static_cast<uint32_t>(__shfl(static_cast<int>(x), lane));
}

// Bitonic sorts over the lanes of a wave, what is ahead in lane 0.  A step keeps, of a pair of lanes, what is ahead in one and the other
// in the other.
__device__ __forceinline__ bool ahead(uint32_t a, uint32_t b) { return a > b; }
__device__ __forceinline__ bool ahead(uint64_t a, uint64_t b) { return a > b; }
template <int M, class X>
__device__ __forceinline__ X exchange(const X& x, bool keep_ahead, int lane) {
  const X other = of_xor<M>(x, lane);
  return keep_ahead == ahead(x, other) ? x : other;
}
template <int SIZE, int M, class X>
__device__ __forceinline__ X steps(X x, int lane) {
  x = exchange<M>(x, ((lane & M) == 0) == ((lane & SIZE) == 0 || SIZE == 64), lane);
  if constexpr (M > 1) x = steps<SIZE, M / 2>(x, lane);
  return x;
}
template <class X>
__device__ __forceinline__ X sorted(X x, int lane) {
  x = steps<2, 1>(x, lane);
  x = steps<4, 2>(x, lane);
  x = steps<8, 4>(x, lane);
  x = steps<16, 8>(x, lane);
  x = steps<32, 16>(x, lane);
  return steps<64, 32>(x, lane);
}
// The 64 ahead of two sorted lists, sorted: the one ahead of each and the opposite of the other are them, as a bitonic sequence.
template <class X>
__device__ __forceinline__ X merged(X x, const X& opposite, int lane) {
  x = ahead(x, opposite) ? x : opposite;
  return steps<64, 32>(x, lane);
}

// ---- rows ---------------------------------------------------------------------------------------------------------------

struct RowArgs {
  const void* logits;        // [rows][V]
  const uint8_t* finished;   // [rows] or nullptr
  uint64_t* best;            // [rows][parts][K]
  double* sums;              // [rows][parts]: of exp(logit - top)
  float* tops;               // [rows][parts]: a whole number above all logits of the part, or what stands for it (see row_kernel)
  long long rows;
  int V, K, parts, part_items;  // items of a part: a multiple of kPiece
};

constexpr int kLaneItems = 8;                 // of a lane, in a piece
constexpr int kPiece = 64 * kLaneItems;
constexpr int kPieces = 2;                    // on their way together

template <class T>
struct Items {
  T x[kLaneItems];
};
// Eight logits from item `first` on; those behind V count as -inf.
template <class T>
__device__ __forceinline__ Items<T> load(const T* row, int first, int V) {
  typedef u32x4_t __attribute__((aligned(2))) word2;
  typedef u32x4_t __attribute__((aligned(4))) word4;
  Items<T> r;
  if (first + kLaneItems <= V) {
    if constexpr (sizeof(T) == 2) {
      const u32x4_t w = *reinterpret_cast<const word2*>(row + first);
      __builtin_memcpy(&r, &w, 16);
    } else {
      const u32x4_t w[2] = {*reinterpret_cast<const word4*>(row + first), *reinterpret_cast<const word4*>(row + first + 4)};
      __builtin_memcpy(&r, w, 32);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kLaneItems; ++i) r.x[i] = first + i < V ? row[first + i] : static_cast<T>(-__builtin_inff());
  }
  return r;
}

template <int M = 1>
__device__ __forceinline__ float greatest_of_wave(float x, int lane) {
  x = fmaxf(x, __uint_as_float(of_xor<M>(__float_as_uint(x), lane)));
  if constexpr (M < 32) x = greatest_of_wave<2 * M>(x, lane);
  return x;
}

// e^(x - top): of the difference, so that a shift of all logits costs nothing, and with log2(e) as two floats.  Errors are those of small
// numbers where the value is large, and of either sign.  (x = top = +inf: NaN.)
__device__ __forceinline__ float exponential(float x, float top) {
  const float d = x - top;
  return __builtin_amdgcn_exp2f(fmaf(d, 1.44269502f, d * 1.92596303e-8f));
}
// e^d for d <= 0 in 64 bits: e^r for what is left of d by whole multiples of ln 2, by its series (r^12 / 12! < 1e-14).
__device__ __forceinline__ double exponential(double d) {
  const double n = rint(d * 1.4426950408889634), r = fma(n, -1.9082149292705877e-10, fma(n, -0.693147180369123816490, d));
  double s = 1.0 / 39916800.0;
  constexpr double kTerms[] = {1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 11; ++i) s = fma(s, r, kTerms[i]);
  return d > -700.0 ? ldexp(s, static_cast<int>(n)) : 0.0;
}

// A wave a part.  The list of the best is sorted over the lanes; a key that is not ahead of the K-th is left out by one
// comparison, so most pieces cost a maximum and their exponentials.  Those that are go through a buffer in LDS, sorted and merged
// by 64.  The K-th is bounded from below by the K-th of the lanes' own greatest, as that many are ahead of it or at it: looked up in the
// first round, the third, and whenever the rounds have doubled (in the first alone, seven in eight of 8300 items' keys that passed were in vain).
// 256 x 8 rows of 16600 bf16 in 25 us (2.8 TB/s), bound by vector instructions, some 18 a logit.
template <class T>
__global__ __launch_bounds__(256) void row_kernel(RowArgs a) {
  __shared__ uint64_t buffers[4][64 + kPiece];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long unit = static_cast<long long>(blockIdx.x) * 4 + wave;
  if (unit >= a.rows * a.parts) return;
  const long long row = unit / a.parts;
  if (a.finished != nullptr && a.finished[row] != 0) return;  // (what it holds is known, see join_kernel)
  const int part = static_cast<int>(unit - row * a.parts), begin = part * a.part_items;
  const int end = begin + a.part_items < a.V ? begin + a.part_items : a.V;
  const T* logits = static_cast<const T*>(a.logits) + row * a.V;
  uint64_t* buffer = buffers[wave];

  uint64_t list = 0;       // (less than every key)
  uint64_t least = 0;      // a key that K or more are ahead of, or at
  int waiting = 0;         // keys in the buffer
  float top = -__builtin_inff();   // greatest logit of the lane
  float above = -__builtin_inff(); // of the wave: what exponentials are taken of differences from, at or above all of its logits
  double sum = 0.0;
  // the last up to 64 of the buffer into the list
  auto take = [&]() {
    const int from = waiting > 64 ? waiting - 64 : 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    list = merged(list, shuffle(sorted(from + lane < waiting ? buffer[from + lane] : uint64_t{0}, lane), 63 - lane), lane);
    const uint64_t kth = shuffle(list, a.K - 1);
    least = kth > least ? kth : least;
    waiting = from;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  };
  Items<T> next[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) next[u] = load(logits, begin + u * kPiece + lane * kLaneItems, end);
  for (int at = begin, round = 0; at < end; at += kPieces * kPiece, ++round) {
    float x[kPieces][kLaneItems], m[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
#pragma unroll
      for (int i = 0; i < kLaneItems; ++i) x[u][i] = static_cast<float>(next[u].x[i]);
      m[u] = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < kLaneItems; ++i) m[u] = fmaxf(m[u], x[u][i]);   // (not the NaNs)
    }
    if (at + kPieces * kPiece < end)
#pragma unroll
      for (int u = 0; u < kPieces; ++u) next[u] = load(logits, at + (kPieces + u) * kPiece + lane * kLaneItems, end);
    float greatest = m[0];
#pragma unroll
    for (int u = 1; u < kPieces; ++u) greatest = fmaxf(greatest, m[u]);
    // the sum, every lane's own; +inf gives no sum (see join_kernel).  What it is relative to rises for the whole wave, by more than 1 beyond the
    // greatest logit, so seldom, and by a factor in 64 bits: one in 32 at every rise would add up over the rounds of a row that rises.
    top = fmaxf(top, greatest);
    if (__ballot(greatest > above) != 0) {
      const float higher = ceilf(greatest_of_wave(greatest, lane)) + 1.0f;
      if (__ballot(above > -__builtin_inff()) != 0) sum *= exponential(static_cast<double>(above) - static_cast<double>(higher));
      above = higher;
    }
    const float against = above > -__builtin_inff() ? above : 0.0f;
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      float e[kLaneItems];
#pragma unroll
      for (int i = 0; i < kLaneItems; ++i) e[i] = exponential(x[u][i], against);
      float s = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      if (__ballot(s != s) != 0) {  // NaNs among them count as nothing
        asm volatile("" ::: "memory");  // (a branch: made ahead of it, this costs as much again)
#pragma unroll
        for (int i = 0; i < kLaneItems; ++i) e[i] = x[u][i] == x[u][i] ? exponential(x[u][i], against) : 0.0f;
        s = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      }
      sum += static_cast<double>(s);
    }
    // the best
    if ((round & (round - 1)) == 0 && round != 1) {
      const uint64_t kth = static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(sorted(in_order(top), lane)), a.K - 1))) << 32;
      least = kth > least ? kth : least;
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      // only where a lane has a key ahead of the K-th
      const float bar = from_order(static_cast<uint32_t>(least >> 32));
      if (__ballot(!(m[u] < bar)) == 0) continue;
      const int first = at + u * kPiece + lane * kLaneItems;
#pragma unroll
      for (int i = 0; i < kLaneItems; ++i) {
        if (__ballot(!(x[u][i] < bar)) == 0) continue;
        const uint64_t key = first + i < end ? key_of(x[u][i], first + i) : 0;
        const bool ahead = key > least;
        const uint64_t votes = __ballot(ahead);
        if (ahead) buffer[waiting + __popcll(votes & ((1ull << lane) - 1))] = key;
        waiting += __popcll(votes);
      }
      while (waiting >= 64) take();
    }
  }
  if (waiting > 0) take();
  if (lane < a.K) a.best[unit * a.K + lane] = list;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
  if (lane == 0) {
    a.sums[unit] = sum;
    a.tops[unit] = above;
  }
}

// ---- joining ------------------------------------------------------------------------------------------------------------

struct JoinArgs {
  const void* logits;
  int dtype;
  const uint64_t* best;
  const double* sums;
  const float* tops;
  const float* scores;       // [B][K]
  const uint8_t* finished;
  float* new_scores;
  int* parents;
  int* tokens;
  int V, K, parts, pad;
  double near;               // see how_near
};

// One candidate: greater total first, then the lower index.
struct Candidate {
  double total;
  uint64_t index;  // beam * V + item
};
__device__ __forceinline__ bool ahead(const Candidate& a, const Candidate& b) {
  return a.total > b.total || (a.total == b.total && a.index < b.index);
}
template <int M>
__device__ __forceinline__ Candidate of_xor(const Candidate& c, int lane) {
  return Candidate{__builtin_bit_cast(double, of_xor<M>(__builtin_bit_cast(uint64_t, c.total), lane)), of_xor<M>(c.index, lane)};
}

constexpr int kJoinThreads = 256;
constexpr int kRowLanes = 16;              // that read a row's sums

// log sum exp of a row in 64 bits, by the whole workgroup; sixteen logits of a thread on their way together.  `top` is their greatest.
// A row of 16600 takes 12 us, one of 120000 65: the memory's latency.
template <class T>
__device__ double sum_of_row(const T* row, int V, double top, double* of_wave) {
  constexpr int kUnroll = 16;
  double sum = 0.0;
  for (int at = threadIdx.x; at < V; at += kUnroll * kJoinThreads) {
    T x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) x[u] = at + u * kJoinThreads < V ? row[at + u * kJoinThreads] : static_cast<T>(-__builtin_inff());
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const float v = static_cast<float>(x[u]);
      sum += v == v ? exponential(static_cast<double>(v) - top) : 0.0;
    }
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = of_wave[0];
#pragma unroll
  for (int w = 1; w < kJoinThreads / 64; ++w) sum += of_wave[w];
  return top + log(sum);
}
__device__ double exact_sum(const JoinArgs& a, long long row, double* of_wave) {
  float top = -__builtin_inff();
  // (the row's greatest itself, the heads of its lists: where it has all of the sum, its total is the score exactly; no key is no number)
  for (int p = threadIdx.x & 63; p < a.parts; p += 64) top = fmaxf(top, from_order(static_cast<uint32_t>(a.best[(row * a.parts + p) * a.K] >> 32)));
  top = greatest_of_wave(top, threadIdx.x & 63);
  const long long at = row * a.V;
  if (a.dtype == COTTEN_F32) return sum_of_row(static_cast<const float*>(a.logits) + at, a.V, top, of_wave);
  if (a.dtype == COTTEN_BF16) return sum_of_row(static_cast<const __bf16*>(a.logits) + at, a.V, top, of_wave);
  return sum_of_row(static_cast<const _Float16*>(a.logits) + at, a.V, top, of_wave);
}

__device__ __forceinline__ Candidate of_lane(const Candidate& c, int lane) {
  return Candidate{__builtin_bit_cast(double, shuffle(__builtin_bit_cast(uint64_t, c.total), lane)), shuffle(c.index, lane)};
}

__device__ __forceinline__ uint32_t of_all(uint32_t bits) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) bits |= static_cast<uint32_t>(__shfl_xor(static_cast<int>(bits), m));
  return bits;
}

// A workgroup a sequence.  First the logarithms of its rows' sums, then the K best of what the parts' lists hold: every wave takes 64
// candidates at a time, the firsts of all lists before the seconds, and where one is ahead of the K-th that it has, sorts them
// and merges them into its own 64; the waves' lists are merged at the end.  256 x 8 beams of two parts in 11 us, 4 x 4 in 6: latency, of one sort after the other.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(JoinArgs a) {
  constexpr int kWaves = kJoinThreads / 64;
  __shared__ double of_row[kMostBeams];                 // what a row adds to its logits
  __shared__ float old_scores[kMostBeams];              // (new_scores may be scores)
  __shared__ uint8_t kind[kMostBeams];
  __shared__ Candidate lists_of_waves[kWaves][64];
  __shared__ double exact[kWaves];
  __shared__ uint32_t unsure;
  enum { kOpen, kEnded, kNothing };
  const int lists = a.K * a.parts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long first_row = static_cast<long long>(blockIdx.x) * a.K;
  const uint64_t* best = a.best + first_row * a.parts * a.K;
  const Candidate none = {-__builtin_inf(), ~0ull};
  for (int k = threadIdx.x / kRowLanes; k < a.K; k += kJoinThreads / kRowLanes) {
    const long long row = first_row + k;
    const int sub = threadIdx.x % kRowLanes;
    const float score = a.scores[row];
    const bool ended = a.finished != nullptr && a.finished[row] != 0;
    double value = static_cast<double>(score);
    if (!ended) {
      float top = -__builtin_inff();
      for (int p = sub; p < a.parts; p += kRowLanes) top = fmaxf(top, a.tops[row * a.parts + p]);
#pragma unroll
      for (int m = 1; m < kRowLanes; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
      double sum = 0.0;
      for (int p = sub; p < a.parts; p += kRowLanes) {
        const double s = a.sums[row * a.parts + p];
        if (!(s == 0.0)) sum += s * exp(static_cast<double>(a.tops[row * a.parts + p]) - static_cast<double>(top));
      }
#pragma unroll
      for (int m = 1; m < kRowLanes; m <<= 1) sum += __shfl_xor(sum, m);
      value -= static_cast<double>(top) + log(sum);
    }
    if (sub == 0) {
      old_scores[k] = score;
      of_row[k] = value;
      // a score or a sum that is not finite leaves a beam no continuation but at -inf
      kind[k] = !(fabs(value) < __builtin_inf()) ? kNothing : ended ? kEnded : kOpen;
    }
  }
  __syncthreads();

  // the n-th of a list.  A beam that ended has one list: the pad item, then the others from the lowest on, at -inf; one without anything
  // has them from 0 on.
  auto candidate = [&](int list, int n, uint64_t key) {
    const int k = list / a.parts;
    const uint64_t base = static_cast<uint64_t>(k) * a.V;
    if (kind[k] == kOpen) {
      if (key == 0) return none;
      return Candidate{static_cast<double>(from_order(static_cast<uint32_t>(key >> 32))) + of_row[k], base + static_cast<uint32_t>(~key)};
    }
    if (list != k * a.parts || n >= a.V) return none;
    if (kind[k] == kNothing) return Candidate{none.total, base + n};
    if (n == 0) return Candidate{of_row[k], base + a.pad};
    return Candidate{none.total, base + (n - 1 < a.pad ? n - 1 : n)};
  };
  for (bool again = false;; again = true) {
    Candidate mine = none, bar = none;       // what a candidate has to be ahead of: the K-th, or as near behind it as sums may be off
    // (lists fall: where no candidate of a wave's lists is ahead, those behind them are not)
    auto take = [&](int list, int n) {
      const Candidate c = n < a.K ? candidate(list, n, best[static_cast<long long>(list) * a.K + n]) : none;
      if (__ballot(ahead(c, bar)) == 0) return false;
      mine = merged(mine, of_lane(sorted(c, lane), 63 - lane), lane);
      bar = Candidate{of_lane(mine, a.K - 1).total - a.near, ~0ull};
      return true;
    };
    if (lists > 64) {
      for (int at = wave * 64; at < lists; at += kJoinThreads) {
        const bool there = at + lane < lists;
        for (int n = 0; n < a.K && take(there ? at + lane : 0, there ? n : a.K); ++n) {
        }
      }
    } else {
      const int ranks = 64 / lists, n = lane / lists, list = lane - n * lists;
      for (int at = wave * ranks; at < a.K && take(list, n < ranks ? at + n : a.K); at += kWaves * ranks) {
      }
    }
    if (lists * a.K > 64) {
      lists_of_waves[wave][lane] = mine;
      __syncthreads();
      if (wave == 0)
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mine = merged(mine, lists_of_waves[w][63 - lane], lane);
    }
    if (wave == 0) {
      const int k = static_cast<int>(mine.index / static_cast<uint64_t>(a.V));
      if (lane < a.K) {
        a.new_scores[first_row + lane] = static_cast<float>(mine.total);
        a.parents[first_row + lane] = k;
        a.tokens[first_row + lane] = static_cast<int>(mine.index - static_cast<uint64_t>(k) * a.V);
      }
      // beams with candidates nearer to each other, or to the last that is taken, than their sums tell apart
      const int before = lane < a.K ? (lane > 0 ? lane - 1 : 0) : a.K - 1;
      const double gap = of_lane(mine, before).total - mine.total;
      const int k_before = __shfl(k, before);
      const uint32_t pair = mine.index != ~0ull && k != k_before && gap < a.near ? (1u << k) | (1u << k_before) : 0u;
      // (equal totals are those of equal rows: they are in order, but stay equal only if both sums are made again)
      uint32_t near = 0u, more = of_all(gap > 0.0 ? pair : 0u);
      // Where the last of the 64 is that near too, others may have found no place (one beam's equal logits can take them all): every beam
      // with a candidate that near behind the last that is taken is looked up in the lists.
      if (!again && __ballot(lane == 63 && mine.index != ~0ull && gap < a.near) != 0) {
        const Candidate last = of_lane(mine, a.K - 1);
        const uint32_t of_last = 1u << __shfl(k, a.K - 1);
        uint32_t crowd = 0u;
        bool differ = false;
        for (int list = lane; list < lists; list += 64) {
          if ((of_last >> (list / a.parts)) & 1u) continue;   // (in order by itself)
          for (int n = 0; n < a.K; ++n) {
            const Candidate c = candidate(list, n, best[static_cast<long long>(list) * a.K + n]);
            if (!(last.total - c.total < a.near)) break;
            if (ahead(last, c)) {
              crowd |= 1u << (list / a.parts);
              differ |= c.total < last.total;
            }
          }
        }
        crowd = of_all(crowd);
        if (crowd != 0u && (more != 0u || __ballot(differ) != 0)) more |= crowd | of_last;
      }
      while (more != near) {
        near = more;
        more |= of_all((pair & near) != 0u ? pair : 0u);
      }
      if (lane == 0) unsure = again ? 0u : near;
    }
    __syncthreads();
    const uint32_t rows = unsure;
    if (rows == 0) return;
    for (int k = 0; k < a.K; ++k) {
      if (!((rows >> k) & 1u) || kind[k] != kOpen) continue;
      const double sum = exact_sum(a, first_row + k, exact);
      if (threadIdx.x == 0) of_row[k] = static_cast<double>(old_scores[k]) - sum;
    }
    __syncthreads();
  }
}

// ---- reordering -----------------------------------------------------------------------------------------------------------

// Beam k of a sequence gets what beam parents[k] had, in place: a thread owns some bytes of all K beams, and loads all that move
// before it stores any.  A beam that stays is neither read nor written; a parent that is none leaves a beam as it is.  256 x 8 beams of
// 64 KB (134 MB) in 28 us, for which the memory-side cache holds much of them.
template <class Word, int MOST>
__global__ __launch_bounds__(256) void reorder_kernel(Word* state, const int* parents, int K, long long words, int blocks) {
  const long long sequence = blockIdx.x / blocks;
  const long long at = static_cast<long long>(blockIdx.x - sequence * blocks) * 256 + threadIdx.x;
  Word* of = state + sequence * K * words;
  const int* from = parents + sequence * K;
  for (long long w = at; w < words; w += static_cast<long long>(blocks) * 256) {
    Word x[MOST];
    uint32_t moves = 0;
#pragma unroll
    for (int k = 0; k < MOST; ++k)
      if (k < K) {
        const int p = from[k];
        if (p >= 0 && p < K && p != k) {
          moves |= 1u << k;
          x[k] = of[p * words + w];
        }
      }
#pragma unroll
    for (int k = 0; k < MOST; ++k)
      if ((moves >> k) & 1u) of[k * words + w] = x[k];
  }
}

template <class Word>
void launch_reorder(void* state, const int* parents, int B, int K, size_t bytes, hipStream_t s) {
  const long long words = static_cast<long long>(bytes / sizeof(Word));
  long long blocks = (words + 255) / 256;
  while (blocks > 1 && blocks * B > (1 << 16)) blocks = (blocks + 1) / 2;
  const dim3 grid(static_cast<unsigned>(blocks * B)), block(256);
  Word* w = static_cast<Word*>(state);
  if (K <= 4) reorder_kernel<Word, 4><<<grid, block, 0, s>>>(w, parents, K, words, static_cast<int>(blocks));
  else if (K <= 8) reorder_kernel<Word, 8><<<grid, block, 0, s>>>(w, parents, K, words, static_cast<int>(blocks));
  else if (K <= 16) reorder_kernel<Word, 16><<<grid, block, 0, s>>>(w, parents, K, words, static_cast<int>(blocks));
  else reorder_kernel<Word, 32><<<grid, block, 0, s>>>(w, parents, K, words, static_cast<int>(blocks));
}

// ---- launches -----------------------------------------------------------------------------------------------------------

bool aligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_shape(int B, int K, int V) {
  if (B < 1 || K < 1 || V < 1 || K > kMostBeams || V >= (1 << 30) || static_cast<long long>(B) * K >= (1ll << 22)) return COTTEN_ERR_BAD_SHAPE;
  return COTTEN_OK;
}

// Totals of two beams nearer than this may be in the wrong order.  A row's logarithm is off by what its exponentials are on the average that
// the sum takes: 2^-23 of the hardware's, and 2^-24 of their exponents by the difference and again by its product with log2(e).  The exponents
// are 2 more than those from the row's greatest at most, which are ln V at most on that average.  Three roundings in a sum of eight by pairs;
// everything after it is in 64 bits.
double how_near(int V) { return 2.0 * (2.0 + 2.0 * (2.0 + std::log(static_cast<double>(V))) + 3.0) / 16777216.0; }

// Waves for a row: enough of them to fill the device, of one round of loads at least; few enough that the join has up to 512 lists.
// 256 x 8 rows of 16600 in 8192 / 4096 / 2048 waves: 44 / 38 / 39 us with the join; 32 x 5 of 120000: 39 / 35 / 32 (before the bar was raised again).
constexpr int kWanted = 4096;
struct Cut {
  int parts, part_items;
  Cut(int B, int K, int V) {
    const long long rows = static_cast<long long>(B) * K, round = kPiece * kPieces;
    const long long rounds = (V + round - 1) / round, most = 512 / K < 64 ? 512 / K : 64;
    long long wanted = (kWanted + rows - 1) / rows;
    wanted = wanted < 1 ? 1 : wanted > most ? most : wanted;
    const long long each = (rounds + wanted - 1) / wanted;
    part_items = static_cast<int>(each * round);
    parts = static_cast<int>((V + static_cast<long long>(part_items) - 1) / part_items);
  }
  size_t units(int B, int K) const { return static_cast<size_t>(B) * K * parts; }
};

}  // namespace
}  // namespace beam
}  // namespace cotten

using namespace cotten::beam;

extern "C" {

size_t cotten_beam_workspace_bytes(int B, int K, int V) {
  if (check_shape(B, K, V) != COTTEN_OK) return 0;
  const size_t units = Cut(B, K, V).units(B, K);
  return units * (K * sizeof(uint64_t) + sizeof(double) + sizeof(float));
}

int cotten_beam_select(const void* logits, const float* scores, const uint8_t* finished, float* new_scores, int32_t* parents,
                       int32_t* tokens, int B, int K, int V, void* stream, const cotten_beam_params* prm) {
  if (prm == nullptr || logits == nullptr || scores == nullptr || new_scores == nullptr || parents == nullptr || tokens == nullptr)
    return COTTEN_ERR_NULL_POINTER;
  if (prm->dtype != COTTEN_F32 && prm->dtype != COTTEN_BF16 && prm->dtype != COTTEN_F16) return COTTEN_ERR_BAD_DTYPE;
  if (int rc = check_shape(B, K, V)) return rc;
  if (finished != nullptr && (prm->pad < 0 || prm->pad >= V)) return COTTEN_ERR_BAD_PARAM;
  if (!aligned(logits, 16) || !aligned(prm->workspace, 16)) return COTTEN_ERR_MISALIGNED;
  if (!aligned(scores, 4) || !aligned(new_scores, 4) || !aligned(parents, 4) || !aligned(tokens, 4)) return COTTEN_ERR_MISALIGNED;
  if (prm->workspace == nullptr || prm->workspace_bytes < cotten_beam_workspace_bytes(B, K, V)) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  const Cut cut(B, K, V);
  const size_t units = cut.units(B, K);
  uint64_t* best = static_cast<uint64_t*>(prm->workspace);
  double* sums = reinterpret_cast<double*>(best + units * K);
  float* tops = reinterpret_cast<float*>(sums + units);
  const RowArgs r{logits, finished, best, sums, tops, static_cast<long long>(B) * K, V, K, cut.parts, cut.part_items};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<unsigned>((units + 3) / 4)), block(256);
  if (prm->dtype == COTTEN_F32) row_kernel<float><<<grid, block, 0, s>>>(r);
  else if (prm->dtype == COTTEN_BF16) row_kernel<__bf16><<<grid, block, 0, s>>>(r);
  else row_kernel<_Float16><<<grid, block, 0, s>>>(r);
  const JoinArgs j{logits, prm->dtype, best, sums, tops, scores, finished, new_scores, parents, tokens, V, K, cut.parts, prm->pad, how_near(V)};
  join_kernel<<<dim3(B), dim3(kJoinThreads), 0, s>>>(j);
  return hipGetLastError() == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

int cotten_beam_reorder(void* state, const int32_t* parents, int B, int K, size_t bytes, void* stream) {
  if (state == nullptr || parents == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (check_shape(B, K, 1) != COTTEN_OK || bytes < 1 || bytes >= (1ull << 40)) return COTTEN_ERR_BAD_SHAPE;
  if (!aligned(parents, 4)) return COTTEN_ERR_MISALIGNED;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (bytes % 16 == 0 && aligned(state, 16)) launch_reorder<u32x4_t>(state, parents, B, K, bytes, s);
  else if (bytes % 4 == 0 && aligned(state, 4)) launch_reorder<uint32_t>(state, parents, B, K, bytes, s);
  else launch_reorder<uint8_t>(state, parents, B, K, bytes, s);
  return hipGetLastError() == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

}  // extern "C"
