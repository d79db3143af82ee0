// A step of a beam search: the best K of the K * V continuations of every sequence's K beams, and the reordering of what
// belongs to the beams.
//
//     total[k, v] = score[k] + logit[k, v] - log sum_v' exp(logit[k, v'])        a beam that ended: score[k] at the pad
//                                                                                 item, -inf elsewhere
//
// The best, the lower k * V + v of equal ones first.  Within a beam the order of the totals is that of the logits, so a row of
// logits is read once, in parts: a wave keeps the K best of its part (value and item) and the sum of the exponentials, and
// one workgroup a sequence joins what the parts of its K rows hold, with totals in 64 bits.
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

__device__ __forceinline__ uint64_t shuffle_xor(uint64_t x, int m) {
  return (static_cast<uint64_t>(static_cast<uint32_t>(__shfl_xor(static_cast<int>(x >> 32), m))) << 32) |
         static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), m));
}
__device__ __forceinline__ uint64_t shuffle(uint64_t x, int lane) {
  return (static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(x >> 32), lane))) << 32) |
         static_cast<uint32_t>(__shfl(static_cast<int>(x), lane));
}

// The 64 keys of a wave, the greatest in lane 0 (bitonic).
__device__ __forceinline__ uint64_t sorted(uint64_t x, int lane) {
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int m = size >> 1; m > 0; m >>= 1) {
      const uint64_t other = shuffle_xor(x, m);
      const bool upper = (lane & m) == 0, falling = (lane & size) == 0 || size == 64;
      x = (upper == falling) == (x > other) ? x : other;
    }
  return x;
}
// The 64 greatest of two sorted lists, sorted: the greater of each and the opposite of the other are them, as a bitonic sequence.
__device__ __forceinline__ uint64_t merged(uint64_t x, uint64_t y, int lane) {
  const uint64_t z = shuffle(y, 63 - lane);
  x = x > z ? x : z;
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    const uint64_t other = shuffle_xor(x, m);
    x = ((lane & m) == 0) == (x > other) ? x : other;
  }
  return x;
}

// ---- rows ---------------------------------------------------------------------------------------------------------------

struct RowArgs {
  const void* logits;        // [rows][V]
  const uint8_t* finished;   // [rows] or nullptr
  uint64_t* best;            // [rows][parts][K]
  double* sums;              // [rows][parts]: of exp(logit - top)
  float* tops;               // [rows][parts]
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

__device__ __forceinline__ float greatest_of_wave(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

// exp(x - top) for x <= top, to about an ulp of 2^-23: the product of the difference with log2(e) is kept as two floats.  (Beyond
// e^-150 it is 0, and where there is no difference of two infinities.)
__device__ __forceinline__ float exponential(float x, float top) {
  const float d = fmaxf(x - top, -150.0f), log2e = 1.44269502f, rest = 1.92596303e-8f;
  const float y = d * log2e;
  const float low = fmaf(d, log2e, -y) + d * rest;
  const float e = __builtin_amdgcn_exp2f(y);
  return fmaf(e * 0.693147182f, low, e);
}

// A wave a part.  The list of the best is sorted over the lanes; a key that is not ahead of the K-th is left out by one
// comparison, so most pieces cost a maximum and their exponentials.  Those that are go through a buffer of 64 in LDS, sorted and merged
// when it is full.
template <class T>
__global__ __launch_bounds__(256) void row_kernel(RowArgs a) {
  __shared__ uint64_t buffers[4][64];
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
  uint64_t least = 0;      // the K-th of the list
  int waiting = 0;         // keys in the buffer
  float top = -__builtin_inff();
  double sum = 0.0;
  auto empty = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    list = merged(list, sorted(lane < waiting ? buffer[lane] : 0, lane), lane);
    least = shuffle(list, a.K - 1);
    waiting = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  };
  Items<T> next[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) next[u] = load(logits, begin + u * kPiece + lane * kLaneItems, end);
  for (int at = begin; at < end; at += kPieces * kPiece) {
    float x[kPieces][kLaneItems];
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int i = 0; i < kLaneItems; ++i) {
        x[u][i] = static_cast<float>(next[u].x[i]);
        x[u][i] = x[u][i] != x[u][i] ? -__builtin_inff() : x[u][i];
      }
    if (at + kPieces * kPiece < end)
#pragma unroll
      for (int u = 0; u < kPieces; ++u) next[u] = load(logits, at + (kPieces + u) * kPiece + lane * kLaneItems, end);
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      float m = x[u][0];
#pragma unroll
      for (int i = 1; i < kLaneItems; ++i) m = fmaxf(m, x[u][i]);
      const int first = at + u * kPiece + lane * kLaneItems;
      // the sum, every lane's own; +inf gives no sum (see join_kernel)
      if (m > top) {
        sum = top > -__builtin_inff() ? sum * static_cast<double>(exponential(top, m)) : 0.0;
        top = m;
      }
      if (top > -__builtin_inff()) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kLaneItems; ++i) s += exponential(x[u][i], top);
        sum += static_cast<double>(s);
      }
      // the best: only where a lane has a key ahead of the K-th
      const float bar = from_order(static_cast<uint32_t>(least >> 32));
      if (__ballot(least == 0 ? first < end : m >= bar) == 0) continue;
#pragma unroll
      for (int i = 0; i < kLaneItems; ++i) {
        const uint64_t key = first + i < end ? key_of(x[u][i], first + i) : 0;
        const bool ahead = key > least;
        const uint64_t votes = __ballot(ahead);
        if (votes == 0) continue;
        const int many = __popcll(votes);
        if (waiting + many > 64) {
          empty();
          // (some may not be ahead any more: they go in all the same, and fall out in the merge)
        }
        if (ahead) buffer[waiting + __popcll(votes & ((1ull << lane) - 1))] = key;
        waiting += many;
      }
    }
  }
  if (waiting > 0) empty();
  if (lane < a.K) a.best[unit * a.K + lane] = list;
  const float all = greatest_of_wave(top);
  double part_sum = sum > 0.0 ? sum * static_cast<double>(exponential(top, all)) : 0.0;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) part_sum += __shfl_xor(part_sum, m);
  if (lane == 0) {
    a.sums[unit] = part_sum;
    a.tops[unit] = all;
  }
}

// ---- joining ------------------------------------------------------------------------------------------------------------

struct JoinArgs {
  const uint64_t* best;
  const double* sums;
  const float* tops;
  const float* scores;       // [B][K]
  const uint8_t* finished;
  float* new_scores;
  int* parents;
  int* tokens;
  int V, K, parts, pad;
};

// One candidate: greater total first, then the lower index.
struct Candidate {
  double total;
  uint64_t index;  // beam * V + item
};
__device__ __forceinline__ bool ahead(const Candidate& a, const Candidate& b) {
  return a.total > b.total || (a.total == b.total && a.index < b.index);
}
__device__ __forceinline__ Candidate shuffle_xor(const Candidate& c, int m) {
  return Candidate{__builtin_bit_cast(double, shuffle_xor(__builtin_bit_cast(uint64_t, c.total), m)), shuffle_xor(c.index, m)};
}

constexpr int kJoinThreads = 256;

// A workgroup a sequence.  First the logarithms of its rows' sums, then K rounds of the greatest of what is left of the parts' lists:
// they are sorted, so a list is represented by its first that was not taken, and a round is one comparison a list.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(JoinArgs a) {
  extern __shared__ int taken[];                        // of every list
  __shared__ double of_row[kMostBeams];                 // what a row adds to its logits
  __shared__ uint8_t kind[kMostBeams];
  __shared__ Candidate winners[kJoinThreads / 64];
  __shared__ int winner_list[kJoinThreads / 64];
  enum { kOpen, kEnded, kNothing };
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long first_row = static_cast<long long>(blockIdx.x) * a.K;
  for (int k = wave; k < a.K; k += kJoinThreads / 64) {
    const long long row = first_row + k;
    const float score = a.scores[row];
    const bool ended = a.finished != nullptr && a.finished[row] != 0;
    double value = static_cast<double>(score);
    if (!ended) {
      float top = -__builtin_inff();
      for (int p = lane; p < a.parts; p += 64) top = fmaxf(top, a.tops[row * a.parts + p]);
      top = greatest_of_wave(top);
      double sum = 0.0;
      for (int p = lane; p < a.parts; p += 64) {
        const double s = a.sums[row * a.parts + p];
        if (s > 0.0) sum += s * exp(static_cast<double>(a.tops[row * a.parts + p]) - static_cast<double>(top));
      }
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
      value -= static_cast<double>(top) + log(sum);
    }
    if (lane == 0) {
      of_row[k] = value;
      // a score or a sum that is not finite leaves a beam no continuation but at -inf
      kind[k] = !(fabs(value) < __builtin_inf()) ? kNothing : ended ? kEnded : kOpen;
    }
  }
  const int lists = a.K * a.parts;
  for (int i = threadIdx.x; i < lists; i += kJoinThreads) taken[i] = 0;
  __syncthreads();

  // the first of a list that was not taken.  A beam that ended has one list: the pad item, then the others from the lowest on, at -inf; one
  // without anything has them from 0 on.
  auto head = [&](int i) {
    const int k = i / a.parts, part = i - k * a.parts, n = taken[i];
    const double none = -__builtin_inf();
    const uint64_t base = static_cast<uint64_t>(k) * a.V;
    if (kind[k] == kOpen) {
      const uint64_t key = n < a.K ? a.best[((first_row + k) * a.parts + part) * a.K + n] : 0;
      if (key == 0) return Candidate{none, ~0ull};
      return Candidate{static_cast<double>(from_order(static_cast<uint32_t>(key >> 32))) + of_row[k], base + static_cast<uint32_t>(~key)};
    }
    if (part != 0 || n >= a.V) return Candidate{none, ~0ull};
    if (kind[k] == kNothing) return Candidate{none, base + n};
    if (n == 0) return Candidate{of_row[k], base + a.pad};
    return Candidate{none, base + (n - 1 < a.pad ? n - 1 : n)};
  };
  for (int round = 0; round < a.K; ++round) {
    Candidate best = {-__builtin_inf(), ~0ull};
    int from = -1;
    for (int i = threadIdx.x; i < lists; i += kJoinThreads) {
      const Candidate c = head(i);
      if (from < 0 || ahead(c, best)) {
        best = c;
        from = i;
      }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const Candidate other = shuffle_xor(best, m);
      const int other_from = __shfl_xor(from, m);
      if (ahead(other, best)) {
        best = other;
        from = other_from;
      }
    }
    if (lane == 0) {
      winners[wave] = best;
      winner_list[wave] = from;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
      for (int w = 1; w < kJoinThreads / 64; ++w)
        if (ahead(winners[w], best)) {
          best = winners[w];
          from = winner_list[w];
        }
      ++taken[from];
      const int k = static_cast<int>(best.index / static_cast<uint64_t>(a.V));
      a.new_scores[first_row + round] = static_cast<float>(best.total);
      a.parents[first_row + round] = k;
      a.tokens[first_row + round] = static_cast<int>(best.index - static_cast<uint64_t>(k) * a.V);
    }
    __syncthreads();
  }
}

// ---- reordering -----------------------------------------------------------------------------------------------------------

// Beam k of a sequence gets what beam parents[k] had, in place: a thread owns some bytes of all K beams, and loads all that move
// before it stores any.  A beam that stays is neither read nor written; a parent that is none leaves a beam as it is.
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

// Waves for a row: enough of them to fill the device, of one round of loads at least.
struct Cut {
  int parts, part_items;
  Cut(int B, int K, int V) {
    const long long rows = static_cast<long long>(B) * K, round = kPiece * kPieces;
    const long long rounds = (V + round - 1) / round;
    long long wanted = (8192 + rows - 1) / rows;
    wanted = wanted < 1 ? 1 : wanted > 256 ? 256 : wanted;
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
  const JoinArgs j{best, sums, tops, scores, finished, new_scores, parents, tokens, V, K, cut.parts, prm->pad};
  join_kernel<<<dim3(B), dim3(kJoinThreads), K * cut.parts * sizeof(int), s>>>(j);
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
