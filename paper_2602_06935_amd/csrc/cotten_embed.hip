// Embedding of item ids, E[b,n] = scale * W[id] + P[offset + n], and its gradient:
//
//     dW[i] = scale * sum over the tokens with id i of dE (in a fixed order)      dP[offset + n] = sum_b dE[b,n]
//
// Everything here moves memory.  The gradient of the table sorts the tokens by id (stable, so a row's sum has one order
// and a call one result) and sums the sorted rows in units of a few tokens, whatever ids they have: a popular item is
// many units, a rare one a part of one, and no workgroup waits for the most popular item.  Up to 8192 tokens are sorted by the
// workgroups that sum them, in one launch.  Sums are fp32, whatever the type, and rounded once, where they are stored.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/cotten_attn.h"

namespace cotten {
namespace embed {
namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// ---- VEC elements of a row ------------------------------------------------------------------------------------------

template <int BYTES>
struct Word;
template <>
struct Word<2> { typedef uint16_t type; };
template <>
struct Word<4> { typedef uint32_t type; };
template <>
struct Word<8> { typedef u32x2_t type; };
template <>
struct Word<16> { typedef u32x4_t type; };

template <class T, int VEC>
struct Vec {
  typedef typename Word<sizeof(T) * VEC>::type word;
  typedef T elems __attribute__((ext_vector_type(VEC)));
  static __device__ __forceinline__ void load(const T* p, float (&x)[VEC]) {
    const word w = *reinterpret_cast<const word*>(p);
    if constexpr (VEC == 1) {
      x[0] = static_cast<float>(__builtin_bit_cast(T, w));
    } else {
      const elems e = __builtin_bit_cast(elems, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = static_cast<float>(e[i]);
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&x)[VEC]) {
    if constexpr (VEC == 1) {
      *reinterpret_cast<word*>(p) = __builtin_bit_cast(word, static_cast<T>(x[0]));
    } else {
      elems e;
#pragma unroll
      for (int i = 0; i < VEC; ++i) e[i] = static_cast<T>(x[i]);
      *reinterpret_cast<word*>(p) = __builtin_bit_cast(word, e);
    }
  }
};

struct Ids {
  const void* ids;
  int wide;       // int64
  int V, padding; // rows of the table; the id that stands for no item (-1: none)
  // the id, or V for a token without a row: padding, or outside the table
  __device__ __forceinline__ uint32_t row(long long i) const {
    const long long id = wide ? static_cast<const long long*>(ids)[i] : static_cast<const int*>(ids)[i];
    return id >= 0 && id < V && id != padding ? static_cast<uint32_t>(id) : static_cast<uint32_t>(V);
  }
};

// ---- forward ----------------------------------------------------------------------------------------------------------

constexpr int kThreads = 256;
constexpr long long kMostBlocks = 1ll << 22;  // of a launch, which has less than 2^32 threads
constexpr int kUnroll = 4;  // pieces of a thread: their ids, then their rows, are on the way together

// A piece is VEC elements; pieces are numbered through the rows of a workgroup's tokens.  Bound by memory: 1024 x 200 rows of
// 256 bf16 (105 MB written, rows of a table of 16600 from cache) in 37 us, 2.9 TB/s written; 128 x 200 x 256 fp32 of 120000 rows
// in 11.3 us, 4.6 TB/s both ways.  Four pieces of a thread in flight; their ids are two dependent trips before the first store.
template <class T, int VEC>
__global__ __launch_bounds__(kThreads) void lookup_kernel(Ids ids, const T* __restrict__ W, const T* __restrict__ P,
                                                          T* __restrict__ E, long long tokens, int N, int D, int pieces,
                                                          int block_tokens, int offset, float scale) {
  const long long first = static_cast<long long>(blockIdx.x) * block_tokens;
  const int rows = static_cast<int>(tokens - first < block_tokens ? tokens - first : block_tokens);
  const uint32_t n0 = static_cast<uint32_t>(first % N);
  const uint32_t end = static_cast<uint32_t>(rows) * pieces;
  for (uint32_t at = threadIdx.x; at < end; at += kThreads * kUnroll) {
    uint32_t row[kUnroll], col[kUnroll], id[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t i = at + u * kThreads;
      row[u] = i / pieces;
      col[u] = (i - row[u] * pieces) * VEC;
      id[u] = i < end ? ids.row(first + row[u]) : ids.V;
    }
    float x[kUnroll][VEC];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (id[u] < static_cast<uint32_t>(ids.V)) {
        Vec<T, VEC>::load(W + static_cast<long long>(id[u]) * D + col[u], x[u]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = 0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (at + u * kThreads >= end) break;
      const long long token = first + row[u];
      float p[VEC] = {};
      if (P != nullptr) Vec<T, VEC>::load(P + static_cast<size_t>(offset + (n0 + row[u]) % static_cast<uint32_t>(N)) * D + col[u], p);
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[u][e] = id[u] < static_cast<uint32_t>(ids.V) ? fmaf(scale, x[u][e], p[e]) : p[e];
      Vec<T, VEC>::store(E + token * D + col[u], x[u]);
    }
  }
}

// ---- sorting tokens by id ------------------------------------------------------------------------------------------------
//
// Least significant digits first, up to 9 bits each (two passes for tables of up to 2^18 rows).  A pass: counts of every
// digit in every block, their sums over the blocks before, and the move, which keeps the order of equal digits: a wave
// takes 64 tokens at a time in order, and a token's place among those with its digit is a count of lanes.  204800 tokens:
// 4.3 us, 4.7 and 7.6 a pass, most of it launch and latency: 1.6 MB move.

constexpr int kDigits = 512;
constexpr int kStrips = 2;                                       // of 64 tokens, per wave of the sort's blocks
constexpr int kBlockTokens = (kThreads / 64) * kStrips * 64;

// The launches of a sort wait more than they move: workgroups behind those of the sort write a share of dW's zeros
// (120000 rows of 256 floats take 17 us by themselves).
struct Zeros {
  unsigned char* at;
  size_t bytes;
  uint32_t sort_blocks;  // workgroups before the first that writes
};
constexpr int kZeroBytes = 64 * 1024;  // of a workgroup

template <int THREADS>
__device__ __forceinline__ bool wrote_zeros(const Zeros& z) {
  if (blockIdx.x < z.sort_blocks) return false;
  const size_t first = static_cast<size_t>(blockIdx.x - z.sort_blocks) * kZeroBytes;
  const size_t end = first + kZeroBytes < z.bytes ? first + kZeroBytes : z.bytes, whole = end & ~size_t{15};
  for (size_t i = first + threadIdx.x * 16; i < whole; i += THREADS * 16) *reinterpret_cast<u32x4_t*>(z.at + i) = u32x4_t{0, 0, 0, 0};
  if (whole + threadIdx.x < end) z.at[whole + threadIdx.x] = 0;
  return true;
}

struct Sort {
  Ids ids;
  const uint32_t* keys;    // of the pass before; nullptr: the ids
  const uint32_t* tokens;
  uint32_t* keys_out;
  uint32_t* tokens_out;
  uint32_t* counts;        // [digit][block], then (after the sums) tokens of that digit in the blocks before
  uint32_t* totals;        // [digit]
  uint32_t n;
  int blocks, shift, bits;
  __device__ __forceinline__ uint32_t key(uint32_t i) const { return keys != nullptr ? keys[i] : ids.row(i); }
};

__global__ __launch_bounds__(kThreads) void count_kernel(Sort s, Zeros z) {
  if (wrote_zeros<kThreads>(z)) return;
  __shared__ uint32_t hist[kDigits];
  for (int d = threadIdx.x; d < kDigits; d += kThreads) hist[d] = 0;
  __syncthreads();
  const uint32_t first = blockIdx.x * kBlockTokens, mask = (1u << s.bits) - 1u;
#pragma unroll
  for (int i = 0; i < kBlockTokens / kThreads; ++i) {
    const uint32_t at = first + i * kThreads + threadIdx.x;
    if (at < s.n) atomicAdd(&hist[(s.key(at) >> s.shift) & mask], 1u);
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d <= mask; d += kThreads) s.counts[static_cast<size_t>(d) * s.blocks + blockIdx.x] = hist[d];
}

// A wave per digit.
__global__ __launch_bounds__(kThreads) void sums_kernel(Sort s, Zeros z) {
  if (wrote_zeros<kThreads>(z)) return;
  const int lane = threadIdx.x & 63;
  const uint32_t d = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (d >= (1u << s.bits)) return;
  uint32_t* row = s.counts + static_cast<size_t>(d) * s.blocks;
  uint32_t before = 0;
  for (int b = 0; b < s.blocks; b += 64) {
    const uint32_t own = b + lane < s.blocks ? row[b + lane] : 0;
    uint32_t x = own;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const uint32_t y = __shfl_up(x, m);
      if (lane >= m) x += y;
    }
    if (b + lane < s.blocks) row[b + lane] = before + x - own;
    before += __shfl(x, 63);
  }
  if (lane == 0) s.totals[d] = before;
}

// Exclusive sums of base[0 ... 511], by kThreads threads; `part`: a word per wave.
__device__ __forceinline__ void exclusive_sums(uint32_t* base, uint32_t* part) {
  static_assert(kThreads == kDigits / 2, "two digits a thread");
  const int t = threadIdx.x, lane = t & 63;
  const uint32_t a = base[2 * t], b = base[2 * t + 1];
  uint32_t x = a + b;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  if (lane == 63) part[t >> 6] = x;
  __syncthreads();
  uint32_t before = x - a - b;
  for (int w = 0; w < (t >> 6); ++w) before += part[w];
  base[2 * t] = before;
  base[2 * t + 1] = before + a;
  __syncthreads();
}

// Tokens to their places: a wave has kStrips times 64 of them.  place[w][d] counts up from where wave w's next token with
// digit d goes.
__global__ __launch_bounds__(kThreads) void move_kernel(Sort s, Zeros z) {
  if (wrote_zeros<kThreads>(z)) return;
  constexpr int kWaves = kThreads / 64;
  __shared__ uint32_t place[kWaves][kDigits], base[kDigits], part[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t mine = blockIdx.x * kBlockTokens + wave * (kStrips * 64) + lane, mask = (1u << s.bits) - 1u;
  uint32_t key[kStrips], token[kStrips];
#pragma unroll
  for (int i = 0; i < kStrips; ++i) {
    const uint32_t at = mine + 64 * i;
    key[i] = at < s.n ? s.key(at) : 0;
    token[i] = at < s.n && s.keys != nullptr ? s.tokens[at] : at;
  }
  for (uint32_t i = threadIdx.x; i < (static_cast<uint32_t>(kWaves) << s.bits); i += kThreads) place[i >> s.bits][i & mask] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kStrips; ++i)
    if (mine + 64 * i < s.n) atomicAdd(&place[wave][(key[i] >> s.shift) & mask], 1u);
  for (uint32_t d = threadIdx.x; d < kDigits; d += kThreads) base[d] = d <= mask ? s.totals[d] : 0;
  __syncthreads();
  exclusive_sums(base, part);
  for (uint32_t d = threadIdx.x; d <= mask; d += kThreads) {
    uint32_t at = base[d] + s.counts[static_cast<size_t>(d) * s.blocks + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t x = place[w][d];
      place[w][d] = at;
      at += x;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kStrips; ++i) {
    const bool on = mine + 64 * i < s.n;
    const uint32_t d = (key[i] >> s.shift) & mask;
    uint64_t same = __ballot(on);
    for (int b = 0; b < s.bits; ++b) {
      const uint64_t set = __ballot((d >> b) & 1u);
      same &= ((d >> b) & 1u) ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1ull));
    uint32_t to = 0;
    if (on) to = place[wave][d] + rank;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    if (on && rank == 0) place[wave][d] = to + __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    if (on) {
      s.keys_out[to] = key[i];
      s.tokens_out[to] = token[i];
    }
  }
}

// ---- sums of sorted rows -------------------------------------------------------------------------------------------------
//
// A unit is kUnit consecutive sorted tokens; lanes of a power of two take its columns.  A row whose tokens all lie in one
// unit is written at once.  One that goes on leaves its sum so far: of the unit that it starts in as the tail, of the
// units after that as their head; join_kernel adds these in order.

// Shorter units are more sums to join, longer ones wait longer for their rows.  Backward without dP, bf16, units of 8 / 16 / 32:
// 1024 x 200 x 256, ids uniform in the logarithm 83 / 71 / 76 us; 512 x 50 x 256 of 120000 rows 38 / 42 / 49; 1024 x 200 x 64 of
// 50 rows 42 / 38 / 40.  sum_kernel for the first, with dP: 40 us for 210 MB of dE (read for either sum), 5.3 TB/s.
constexpr int kUnit = 16;

struct Rows {
  const uint32_t* keys;
  const uint32_t* tokens;
  uint32_t n;
  int V, D, lanes;          // lanes: of a row, a power of two
  uint32_t units;
  float* heads;             // [unit][D]
  float* tails;
  float scale;
};

constexpr int kSumThreads = 512;

// dP, by the workgroups of sum_kernel behind its units.  dE is a matrix of B rows and N * D columns here, and dP the sums of
// its columns.  A workgroup has `lanes` pieces of columns, and its lane groups deal the rows of its part out among them;
// workgroups behind these write the zeros of positions that no token has, kZeroBytes each (16384 x 1 x 256 fp32: 36 us for a table
// of 4096 positions as for one of 8).  Few columns of many rows are cut into parts (four or more, of at least kPartRows
// rows) until there are kParts workgroups, and join_positions_kernel adds the parts.  Whole backward, fp32, D = 256, in
// parts / in one: 65536 x 1: 55 / 631 us; 16384 x 4: 51 / 182 us.
template <class T>
struct Positions {
  T* dP;           // nullptr: not wanted
  float* partial;  // [part][N * D]
  size_t width, start, total;  // columns: N * D, those before them, all of dP
  uint32_t B, lanes, parts, blocks;  // blocks: workgroups of a part
};
constexpr int kParts = 256, kPartRows = 64, kPartLanes = 64;

template <class T, int VEC>
__device__ __forceinline__ void sum_positions(const Positions<T>& p, const T* __restrict__ dE, uint32_t index, float* shared) {
  if (index >= p.parts * p.blocks) {
    const size_t first = static_cast<size_t>(index - p.parts * p.blocks) * (kZeroBytes / sizeof(T)), rest = p.total - p.width;
    const size_t end = first + kZeroBytes / sizeof(T) < rest ? first + kZeroBytes / sizeof(T) : rest;
    const float zeros[VEC] = {};
    for (size_t i = first + threadIdx.x * VEC; i < end; i += kSumThreads * VEC)
      Vec<T, VEC>::store(p.dP + (i < p.start ? i : i + p.width), zeros);
    return;
  }
  const uint32_t groups = kSumThreads / p.lanes, group = threadIdx.x / p.lanes, part = index / p.blocks;
  const size_t c = (static_cast<size_t>(index - part * p.blocks) * p.lanes + threadIdx.x % p.lanes) * VEC;
  const bool inside = c < p.width;
  const uint32_t share = (p.B + p.parts - 1) / p.parts, end = (part + 1) * share < p.B ? (part + 1) * share : p.B;
  const uint32_t first = part * share + group, rows = first < end ? (end - first + groups - 1) / groups : 0;
  const T* from = dE + first * p.width + c;
  const size_t step = groups * p.width;
  float sum[VEC] = {};
  if (inside) {
    constexpr int kAhead = 8;  // rows on the way together
    uint32_t i = 0;
    for (; i + kAhead <= rows; i += kAhead, from += kAhead * step) {
      float x[kAhead][VEC];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) Vec<T, VEC>::load(from + u * step, x[u]);
      __builtin_amdgcn_sched_barrier(0);  // (the compiler would wait for each before the next)
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += x[u][e];
    }
    for (; i < rows; ++i, from += step) {
      float x[VEC];
      Vec<T, VEC>::load(from, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += x[e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) shared[e * kSumThreads + threadIdx.x] = sum[e];
  __syncthreads();
  for (uint32_t half = groups / 2; half > 0; half /= 2) {
    if (group < half)
#pragma unroll
      for (int e = 0; e < VEC; ++e) shared[e * kSumThreads + threadIdx.x] += shared[e * kSumThreads + threadIdx.x + half * p.lanes];
    __syncthreads();
  }
  if (group == 0 && inside) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[e] = shared[e * kSumThreads + threadIdx.x];
    if (p.parts == 1) {
      Vec<T, VEC>::store(p.dP + p.start + c, sum);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) p.partial[part * p.width + c + e] = sum[e];
    }
  }
}

// A lane per column, a wave per share of the parts.
template <class T>
__global__ __launch_bounds__(kSumThreads) void join_positions_kernel(Positions<T> p) {
  constexpr int kWaves = kSumThreads / 64;
  __shared__ float shared[kWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t c = static_cast<size_t>(blockIdx.x) * 64 + lane;
  float sum = 0.0f;
  if (c < p.width)
#pragma unroll 8
    for (uint32_t i = wave; i < p.parts; i += kWaves) sum += p.partial[i * p.width + c];
  shared[wave][lane] = sum;
  __syncthreads();
  if (wave > 0 || c >= p.width) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sum += shared[w][lane];
  p.dP[p.start + c] = static_cast<T>(sum);
}

template <class T, int VEC>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(Rows s, const T* __restrict__ dE, T* __restrict__ dW, Positions<T> p,
                                                          uint32_t unit_blocks) {
  __shared__ float part[kSumThreads * VEC];
  if (blockIdx.x >= unit_blocks) {
    if (blockIdx.y == 0) sum_positions<T, VEC>(p, dE, blockIdx.x - unit_blocks, part);
    return;
  }
  const uint32_t unit = blockIdx.x * (kSumThreads / s.lanes) + threadIdx.x / s.lanes;
  const int col = (blockIdx.y * s.lanes + threadIdx.x % s.lanes) * VEC;
  if (unit >= s.units || col >= s.D) return;
  const uint32_t first = unit * kUnit, end = first + kUnit < s.n ? first + kUnit : s.n;
  const uint32_t V = s.V;
  uint32_t key[kUnit + 1], token[kUnit];
#pragma unroll
  for (int i = 0; i < kUnit; ++i) {
    key[i] = first + i < end ? s.keys[first + i] : V;
    token[i] = first + i < end ? s.tokens[first + i] : 0;
  }
  key[kUnit] = end < s.n ? s.keys[end] : V;
  if (key[0] == V) return;  // tokens without a row are the last
  const uint32_t before = first > 0 ? s.keys[first - 1] : V;
  bool begun = before != key[0];  // the present row starts in this unit
  float sum[VEC] = {};
  constexpr int kAhead = 8;  // rows on the way together
#pragma unroll
  for (int half = 0; half < kUnit; half += kAhead) {
    float x[kAhead][VEC];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (key[half + i] != V) {
        Vec<T, VEC>::load(dE + static_cast<size_t>(token[half + i]) * s.D + col, x[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t k = key[half + i], next = key[half + i + 1];
      if (k == V) continue;
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += x[i][e];
      const bool ends = next != k, last = half + i == kUnit - 1;
      if (!ends && !last) continue;
      if (ends && begun) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] *= s.scale;
        Vec<T, VEC>::store(dW + static_cast<size_t>(k) * s.D + col, sum);
      } else {
        float* to = (begun ? s.tails : s.heads) + static_cast<size_t>(unit) * s.D + col;
#pragma unroll
        for (int e = 0; e < VEC; ++e) to[e] = sum[e];
      }
      begun = true;
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
    }
  }
}

// A wave per unit: where a row starts in it and goes on, its tail and the heads of the units that it goes on in.  Rows of
// more than kMostHeads are shared by the workgroup's waves afterwards (4 or 64 instead of 16: within 5 % everywhere).  10 us
// for the 12800 units of 1024 x 200 tokens of 256 bf16.
constexpr int kJoinWaves = 16, kMostHeads = 16;

template <class T, int VEC>
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(Rows s, T* __restrict__ dW) {
  __shared__ uint32_t long_heads[kJoinWaves];
  __shared__ float part[kJoinWaves][64 * VEC];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t V = s.V, first_unit = blockIdx.x * kJoinWaves;
  const uint32_t unit = first_unit + wave, first = unit * kUnit, next = first + kUnit;
  uint32_t heads = 0, key = V;
  if (unit < s.units && next < s.n) {
    key = s.keys[next - 1];
    const uint32_t after = s.keys[next], begin = s.keys[first], before = first > 0 ? s.keys[first - 1] : V;
    const bool starts = !(begin == key && before == key);
    if (key != V && after == key && starts) {
      // units whose first token has the key: they follow one another, so where the last of `stride` has it, all have
      auto all_have = [&](uint32_t stride) {
        const uint32_t u = unit + heads + (lane + 1) * stride;
        const uint64_t same = __ballot(u < s.units && s.keys[u < s.units ? u * kUnit : 0] == key);
        const int run = same == ~0ull ? 64 : __ffsll(static_cast<long long>(~same)) - 1;
        heads += run * stride;
        return run == 64;
      };
      if (all_have(1)) {
        while (all_have(4096)) {
        }
        all_have(64);  // (fewer than 4096 are left, then fewer than 64)
        all_have(1);
      }
    }
  }
  if (lane == 0) long_heads[wave] = heads > kMostHeads ? heads : 0;
  if (heads > 0 && heads <= kMostHeads) {
    for (int col = lane * VEC; col < s.D; col += 64 * VEC) {
      float sum[VEC];
      Vec<float, VEC>::load(s.tails + static_cast<size_t>(unit) * s.D + col, sum);
#pragma unroll 4
      for (uint32_t i = 1; i <= heads; ++i) {
        float x[VEC];
        Vec<float, VEC>::load(s.heads + static_cast<size_t>(unit + i) * s.D + col, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += x[e];
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] *= s.scale;
      Vec<T, VEC>::store(dW + static_cast<size_t>(key) * s.D + col, sum);
    }
  }
  __syncthreads();
  for (int w = 0; w < kJoinWaves; ++w) {
    const uint32_t all = long_heads[w];
    if (all == 0) continue;
    const uint32_t owner = first_unit + w, share = (all + kJoinWaves) / kJoinWaves;
    // partial sums 0 (the tail) ... `all`, a contiguous share for each wave
    const uint32_t from = wave * share, to = from + share < all + 1 ? from + share : all + 1;
    for (int c0 = 0; c0 < s.D; c0 += 64 * VEC) {
      const int col = c0 + lane * VEC;
      float sum[VEC] = {};
      if (col < s.D) {
#pragma unroll 8
        for (uint32_t i = from; i < to; ++i) {
          float x[VEC];
          Vec<float, VEC>::load((i == 0 ? s.tails : s.heads) + static_cast<size_t>(owner + i) * s.D + col, x);
#pragma unroll
          for (int e = 0; e < VEC; ++e) sum[e] += x[e];
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) part[wave][lane * VEC + e] = sum[e];
      __syncthreads();
      if (wave == 0 && col < s.D) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          float x = 0.0f;
          for (int i = 0; i < kJoinWaves; ++i) x += part[i][lane * VEC + e];
          sum[e] = x * s.scale;
        }
        Vec<T, VEC>::store(dW + static_cast<size_t>(s.keys[(owner + 1) * kUnit]) * s.D + col, sum);
      }
      __syncthreads();
    }
  }
}

// ---- few tokens: everything in one launch -----------------------------------------------------------------------------------
//
// A workgroup has a share of the table's rows to write zeros to, where no token has them: `rows_of_block` that follow one
// another.  And it has as many rows to sum, dealt out one by one (popular ids tend to be neighbours): it picks their tokens out
// of all ids, in order, sorts them by row and token in LDS, and sums them, a lane group per row, or the whole workgroup for a
// row of more than kUnit.  One launch instead of five to eight, and every workgroup reads all ids.  Whole backward, bf16, so /
// sorted as below (host time: 8): 80 tokens, 3700 rows of 64, 8.0 / 14.5 us;  2000 tokens 8.1 / 19.4;  8000 tokens 13 / 30, and
// with ids uniform in the logarithm 25 / 31;  8000 of 120000 rows of 256 29 / 40.  (8000 tokens with such
// ids lose at rows of 300, which go in 8-byte pieces: 50 rows 40 / 25, 700 41 / 33, 30000 39 / 35; and at 8 rows of 256, 41 / 22.)

constexpr int kDirectTokens = 8192, kFewTokens = 2048;  // (with 2048 a workgroup needs half the LDS, and fewer steps)

template <class T, int VEC, int TOKENS>
__global__ __launch_bounds__(kSumThreads) void direct_kernel(Ids ids, Rows s, const T* __restrict__ dE, T* __restrict__ dW,
                                                             uint32_t rows_of_block, uint32_t row_blocks, Positions<T> p) {
  __shared__ float part[kSumThreads * VEC];
  __shared__ uint32_t list[TOKENS], long_rows[TOKENS / kUnit], counts[TOKENS / 64], long_count, all;
  __shared__ uint32_t taken[kZeroBytes / 2 / 32];  // a bit per row of the share
  if (blockIdx.x >= row_blocks) {
    if (blockIdx.y == 0) sum_positions<T, VEC>(p, dE, blockIdx.x - row_blocks, part);
    return;
  }
  constexpr int kTokenBits = 13, kSteps = TOKENS / kSumThreads, kWaves = kSumThreads / 64, kAhead = 8;
  static_assert(TOKENS <= 1 << kTokenBits, "an entry is a row of the block and a token");
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t first_row = blockIdx.x * rows_of_block, left = s.V - first_row, rows = left < rows_of_block ? left : rows_of_block;
  for (uint32_t i = tid; i * 32 < rows; i += kSumThreads) taken[i] = 0;
  if (tid == 0) long_count = 0;
  uint32_t row[kSteps], at[kSteps];
  bool mine[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint32_t token = i * kSumThreads + tid;
    row[i] = token < s.n ? ids.row(token) : static_cast<uint32_t>(s.V);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint32_t r = row[i] - first_row;  // (V and smaller ones: beyond `rows`, as unsigned)
    if (r < rows) atomicOr(&taken[r / 32], 1u << (r % 32));
    const uint32_t q = row[i] / row_blocks;
    mine[i] = row[i] - q * row_blocks == blockIdx.x && row[i] < static_cast<uint32_t>(s.V);
    row[i] = q;
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint64_t in = __ballot(mine[i]);
    at[i] = __popcll(in & ((1ull << lane) - 1ull));
    if (lane == 0) counts[i * kWaves + wave] = __popcll(in);
  }
  __syncthreads();
  if (blockIdx.y == 0) {
    const float zeros[VEC] = {};
    T* const out = dW + static_cast<size_t>(first_row) * s.D;
    const uint32_t of_row = static_cast<uint32_t>(s.D) / VEC, pieces = rows * of_row;
    for (uint32_t i = tid; i < pieces; i += kSumThreads) {
      const uint32_t r = i / of_row;
      if (!((taken[r / 32] >> (r % 32)) & 1u)) Vec<T, VEC>::store(out + static_cast<size_t>(i) * VEC, zeros);
    }
  }
  if (wave == kWaves - 1) {  // sums of the counts before each
    constexpr int kOfLane = (kSteps * kWaves + 63) / 64;
    uint32_t own[kOfLane], x = 0;
#pragma unroll
    for (int i = 0; i < kOfLane; ++i) {
      const uint32_t k = lane * kOfLane + i;
      own[i] = k < kSteps * kWaves ? counts[k] : 0;
      x += own[i];
    }
    uint32_t before = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(before, d);
      if (lane >= d) before += y;
    }
    if (lane == 63) all = before;
    before -= x;
#pragma unroll
    for (int i = 0; i < kOfLane; ++i) {
      const uint32_t k = lane * kOfLane + i;
      if (k < kSteps * kWaves) counts[k] = before;
      before += own[i];
    }
  }
  __syncthreads();
  const uint32_t m = all;
  if (m == 0) return;
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (mine[i]) list[counts[i * kWaves + wave] + at[i]] = (row[i] << kTokenBits) | (i * kSumThreads + tid);
  uint32_t size = 1;
  while (size < m) size *= 2;
  for (uint32_t i = m + tid; i < size; i += kSumThreads) list[i] = ~0u;
  __syncthreads();
  for (uint32_t k = 2; k <= size && rows_of_block > 1; k *= 2)  // (a bitonic network)
    for (uint32_t j = k / 2; j > 0; j /= 2) {
      for (uint32_t t = tid; t < size / 2; t += kSumThreads) {
        const uint32_t lo = 2 * t - (t & (j - 1)), hi = lo + j, a = list[lo], b = list[hi];
        if ((a > b) == ((lo & k) == 0)) {
          list[lo] = b;
          list[hi] = a;
        }
      }
      __syncthreads();
    }

  const uint32_t groups = kSumThreads / s.lanes, group = tid / s.lanes, col = (blockIdx.y * s.lanes + tid % s.lanes) * VEC;
  const bool inside = col < static_cast<uint32_t>(s.D);
  auto row_of = [&](uint32_t e) { return list[e] >> kTokenBits; };
  auto token_of = [&](uint32_t e) { return list[e] & ((1u << kTokenBits) - 1u); };
  auto place_of = [&](uint32_t r) { return dW + (static_cast<size_t>(r) * row_blocks + blockIdx.x) * s.D; };
  // entries e, e + step ... before `end` of a row, in order
  auto add = [&](float(&sum)[VEC], uint32_t e, uint32_t end, uint32_t step) {
    const T* const from = dE + col;
    for (; e + (kAhead - 1) * step < end; e += kAhead * step) {
      float x[kAhead][VEC];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) Vec<T, VEC>::load(from + static_cast<size_t>(token_of(e + u * step)) * s.D, x[u]);
      __builtin_amdgcn_sched_barrier(0);  // (all on the way before the first is waited for)
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int c = 0; c < VEC; ++c) sum[c] += x[u][c];
    }
    if (e >= end) return;
    float x[kAhead - 1][VEC];
#pragma unroll
    for (int u = 0; u < kAhead - 1; ++u)  // (those beyond the end: the first of these once more)
      Vec<T, VEC>::load(from + static_cast<size_t>(token_of(e + u * step < end ? e + u * step : e)) * s.D, x[u]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < kAhead - 1; ++u)
#pragma unroll
      for (int c = 0; c < VEC; ++c) sum[c] += e + u * step < end ? x[u][c] : 0.0f;
  };
  for (uint32_t e = group; e < m; e += groups) {
    const uint32_t r = row_of(e);
    if (e > 0 && row_of(e - 1) == r) continue;
    if (e + kUnit < m && row_of(e + kUnit) == r) {
      if (tid % s.lanes == 0) long_rows[atomicAdd(&long_count, 1u)] = e;
      continue;
    }
    uint32_t end = e + 1;
    while (end < m && row_of(end) == r) ++end;
    if (inside) {
      float sum[VEC] = {};
      add(sum, e, end, 1);
#pragma unroll
      for (int c = 0; c < VEC; ++c) sum[c] *= s.scale;
      Vec<T, VEC>::store(place_of(r) + col, sum);
    }
  }
  __syncthreads();
  for (uint32_t q = 0; q < long_count; ++q) {
    const uint32_t e = long_rows[q], r = row_of(e);
    uint32_t end = e + kUnit, beyond = m;  // the last entry of the row is before `beyond`, `end` is one of it
    while (end + 1 < beyond) {
      const uint32_t middle = (end + beyond) / 2;
      if (row_of(middle) == r) end = middle;
      else beyond = middle;
    }
    float sum[VEC] = {};
    if (inside) add(sum, e + group, beyond, groups);
#pragma unroll
    for (int c = 0; c < VEC; ++c) part[c * kSumThreads + tid] = sum[c];
    __syncthreads();
    for (uint32_t half = groups / 2; half > 0; half /= 2) {
      if (group < half)
#pragma unroll
        for (int c = 0; c < VEC; ++c) part[c * kSumThreads + tid] += part[c * kSumThreads + tid + half * s.lanes];
      __syncthreads();
    }
    if (group == 0 && inside) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) sum[c] = part[c * kSumThreads + tid] * s.scale;
      Vec<T, VEC>::store(place_of(r) + col, sum);
    }
    __syncthreads();
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int key_bits(int V) {  // of 0 ... V
  int bits = 1;
  while (V >> bits) ++bits;
  return bits;
}

// Where things are in the workspace, in 4-byte words.
struct Layout {
  uint32_t blocks, units;
  int passes, digit_bits;
  size_t list, counts, sums, positions, words;  // list: of each of the four lists
  Layout(int B, int N, int D, int V) {
    const long long n = static_cast<long long>(B) * N;
    blocks = static_cast<uint32_t>((n + kBlockTokens - 1) / kBlockTokens);
    units = static_cast<uint32_t>((n + kUnit - 1) / kUnit);
    const int bits = key_bits(V);
    passes = (bits + 8) / 9;
    digit_bits = (bits + passes - 1) / passes;
    list = (static_cast<size_t>(n) + 3) & ~size_t{3};
    counts = static_cast<size_t>(kDigits) * blocks + kDigits;
    sums = (static_cast<size_t>(units) * D + 3) & ~size_t{3};
    // (kParts workgroups of kPartLanes pieces of up to 8 columns, if rows are in parts)
    const size_t shares = (static_cast<size_t>(B) + kPartRows - 1) / kPartRows, of_all = shares * N * D, most = kParts * kPartLanes * 8;
    positions = shares == 1 ? 0 : of_all < most ? of_all : most;
    words = 4 * list + counts + 2 * sums + positions;
  }
};

// The widest pieces that rows consist of.
int piece_bytes(int D, int elem) {
  int b = 16;
  while ((static_cast<long long>(D) * elem) % b) b /= 2;
  return b;
}
int lanes_of(int pieces) {
  int l = 1;
  while (l < pieces && l < 64) l *= 2;
  return l;
}

// f(Vec<T, VEC> tag) for the pieces of D elements of a type
template <class T, int VEC>
struct Tag {
  typedef T type;
  static constexpr int vec = VEC;
};
template <class T, class F>
void by_piece(int D, F&& f) {
  const int vec = piece_bytes(D, sizeof(T)) / static_cast<int>(sizeof(T));
  if (vec == 8) {
    if constexpr (sizeof(T) == 2) f(Tag<T, 8>());
  } else if (vec == 4) {
    f(Tag<T, 4>());
  } else if (vec == 2) {
    f(Tag<T, 2>());
  } else {
    f(Tag<T, 1>());
  }
}
template <class F>
void by_type(int dtype, int D, F&& f) {
  if (dtype == COTTEN_F32) by_piece<float>(D, f);
  else if (dtype == COTTEN_BF16) by_piece<__bf16>(D, f);
  else by_piece<_Float16>(D, f);
}

int check(const void* ids, int B, int N, int D, int V, const cotten_embed_params* prm, bool positions) {
  if (prm == nullptr || ids == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (prm->dtype != COTTEN_F32 && prm->dtype != COTTEN_BF16 && prm->dtype != COTTEN_F16) return COTTEN_ERR_BAD_DTYPE;
  if (prm->id_bytes != 4 && prm->id_bytes != 8) return COTTEN_ERR_BAD_DTYPE;
  if (B < 1 || N < 1 || D < 1 || V < 1) return COTTEN_ERR_BAD_SHAPE;
  if (D > 65536 || static_cast<long long>(B) * N >= (1ll << 31) || V >= (1 << 30)) return COTTEN_ERR_BAD_SHAPE;
  if (positions && (prm->position_offset < 0 || prm->positions < 1 ||
                    static_cast<long long>(prm->position_offset) + N > prm->positions))
    return COTTEN_ERR_BAD_SHAPE;
  if (!std::isfinite(prm->scale)) return COTTEN_ERR_BAD_PARAM;
  if (reinterpret_cast<uintptr_t>(ids) & (prm->id_bytes - 1)) return COTTEN_ERR_MISALIGNED;
  if (!aligned16(prm->workspace)) return COTTEN_ERR_MISALIGNED;
  return COTTEN_OK;
}

}  // namespace
}  // namespace embed
}  // namespace cotten

using namespace cotten::embed;

extern "C" {

size_t cotten_embed_workspace_bytes(int B, int N, int D, int V) {
  if (B < 1 || N < 1 || D < 1 || V < 1 || D > 65536 || static_cast<long long>(B) * N >= (1ll << 31) || V >= (1 << 30)) return 0;
  return Layout(B, N, D, V).words * 4;
}

int cotten_embed_fwd(const void* ids, const void* W, const void* P, void* E, int B, int N, int D, int V, void* stream,
                     const cotten_embed_params* params) {
  if (W == nullptr || E == nullptr) return COTTEN_ERR_NULL_POINTER;
  if (int rc = check(ids, B, N, D, V, params, P != nullptr)) return rc;
  if (!aligned16(W) || !aligned16(P) || !aligned16(E)) return COTTEN_ERR_MISALIGNED;
  const Ids of{ids, params->id_bytes == 8, V, params->padding_idx};
  const long long tokens = static_cast<long long>(B) * N;
  by_type(params->dtype, D, [&](auto tag) {
    typedef typename decltype(tag)::type T;
    constexpr int VEC = decltype(tag)::vec;
    const int pieces = D / VEC;
    long long block_tokens = kThreads * kUnroll / pieces;
    if (block_tokens < 1) block_tokens = 1;
    const long long fewest = (tokens + kMostBlocks - 1) / kMostBlocks;  // (more than the above for 2^31 pieces only)
    if (block_tokens < fewest) block_tokens = fewest;
    lookup_kernel<T, VEC><<<dim3(static_cast<uint32_t>((tokens + block_tokens - 1) / block_tokens)), dim3(kThreads), 0,
                            static_cast<hipStream_t>(stream)>>>(
        of, static_cast<const T*>(W), static_cast<const T*>(P), static_cast<T*>(E), tokens, N, D, pieces, static_cast<int>(block_tokens),
        params->position_offset, params->scale);
  });
  return hipGetLastError() == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

int cotten_embed_bwd(const void* ids, const void* dE, void* dW, void* dP, int B, int N, int D, int V, void* stream,
                     const cotten_embed_params* params) {
  if (dE == nullptr || (dW == nullptr && dP == nullptr)) return COTTEN_ERR_NULL_POINTER;
  if (int rc = check(ids, B, N, D, V, params, dP != nullptr)) return rc;
  if (!aligned16(dE) || !aligned16(dW) || !aligned16(dP)) return COTTEN_ERR_MISALIGNED;
  const long long n = static_cast<long long>(B) * N;
  const Layout at(B, N, D, V);
  const int elem = params->dtype == COTTEN_F32 ? 4 : 2, vec = piece_bytes(D, elem) / elem, lanes_of_row = lanes_of(D / vec);
  if (dP != nullptr && params->positions > kMostBlocks) return COTTEN_ERR_BAD_SHAPE;
  if (dW != nullptr && n > (1ll << 29)) return COTTEN_ERR_BAD_SHAPE;
  const bool direct = dW != nullptr && n <= kDirectTokens;
  const size_t row = static_cast<size_t>(D) * elem, table = V * row;
  // what sums dW: of the one launch, at least 512 workgroups, if there are rows for them, and more for kZeroBytes of zeros each
  const size_t by_bytes = kZeroBytes / row, by_rows = (static_cast<size_t>(V) + 511) / 512;
  const uint32_t of_rows = static_cast<uint32_t>(by_bytes < 1 ? 1 : by_bytes < by_rows ? by_bytes : by_rows);
  const uint32_t of_block = kSumThreads / lanes_of_row;
  const uint32_t table_blocks = dW == nullptr ? 0 : direct ? (V + of_rows - 1) / of_rows : (at.units + of_block - 1) / of_block;
  uint32_t lanes = kSumThreads, parts = 0, columns = 0;  // of the sums for dP: see Positions
  size_t position_blocks = 0;
  if (dP != nullptr) {
    while (lanes > kPartLanes && kSumThreads / lanes < static_cast<uint32_t>(B)) lanes /= 2;
    const size_t all_columns = (static_cast<size_t>(N) * (D / vec) + lanes - 1) / lanes;
    const size_t shares = (static_cast<size_t>(B) + kPartRows - 1) / kPartRows, most = kParts / all_columns;
    parts = static_cast<uint32_t>(shares < most ? shares : most);
    if (parts < 4) parts = 1;
    columns = static_cast<uint32_t>(all_columns);
    position_blocks = parts * all_columns + (static_cast<size_t>(params->positions - N) * row + kZeroBytes - 1) / kZeroBytes;
    if (parts > 1 && (params->workspace == nullptr || params->workspace_bytes < at.words * 4)) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  }
  if (dW != nullptr && (params->workspace == nullptr || params->workspace_bytes < at.words * 4)) return COTTEN_ERR_WORKSPACE_TOO_SMALL;
  // a launch has less than 2^32 threads (the sort's write a share of the zeros each)
  if (table_blocks + position_blocks >= (1ull << 32) / kSumThreads || (dW != nullptr && table / kZeroBytes >= (1ull << 24)))
    return COTTEN_ERR_BAD_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err = hipSuccess;
  Rows rows{};
  rows.V = V;
  rows.D = D;
  rows.lanes = lanes_of_row;
  if (dW != nullptr) {
    rows.n = static_cast<uint32_t>(n);
    rows.scale = params->scale;
  }
  if (dW != nullptr && !direct) {
    uint32_t* w = static_cast<uint32_t*>(params->workspace);
    uint32_t *keys[2] = {w, w + 2 * at.list}, *tokens[2] = {w + at.list, w + 3 * at.list};
    Sort sort{};
    sort.ids = Ids{ids, params->id_bytes == 8, V, params->padding_idx};
    sort.counts = w + 4 * at.list;
    sort.totals = sort.counts + static_cast<size_t>(kDigits) * at.blocks;
    sort.n = static_cast<uint32_t>(n);
    sort.blocks = at.blocks;
    const int bits = key_bits(V), last = (at.passes - 1) & 1;
    // every launch of the sort with its share of the zeros
    const size_t launches = 3 * at.passes;
    const size_t share = ((table + launches - 1) / launches + kZeroBytes - 1) / kZeroBytes * kZeroBytes;
    size_t written = 0;
    auto with_zeros = [&](uint32_t blocks, Zeros* z) {
      const size_t bytes = table - written < share ? table - written : share;
      *z = Zeros{static_cast<unsigned char*>(dW) + written, bytes, blocks};
      written += bytes;
      return dim3(blocks + static_cast<uint32_t>((bytes + kZeroBytes - 1) / kZeroBytes));
    };
    Zeros z;
    for (int p = 0; p < at.passes; ++p) {
      sort.shift = p * at.digit_bits;
      sort.bits = bits - sort.shift < at.digit_bits ? bits - sort.shift : at.digit_bits;
      sort.keys = p == 0 ? nullptr : keys[(p - 1) & 1];
      sort.tokens = p == 0 ? nullptr : tokens[(p - 1) & 1];
      sort.keys_out = keys[p & 1];
      sort.tokens_out = tokens[p & 1];
      dim3 grid = with_zeros(at.blocks, &z);
      count_kernel<<<grid, dim3(kThreads), 0, s>>>(sort, z);
      grid = with_zeros(((1 << sort.bits) + kThreads / 64 - 1) / (kThreads / 64), &z);
      sums_kernel<<<grid, dim3(kThreads), 0, s>>>(sort, z);
      grid = with_zeros(at.blocks, &z);
      move_kernel<<<grid, dim3(kThreads), 0, s>>>(sort, z);
    }
    err = hipGetLastError();
    rows.keys = keys[last];
    rows.tokens = tokens[last];
    rows.units = at.units;
    rows.heads = reinterpret_cast<float*>(w + 4 * at.list + at.counts);
    rows.tails = rows.heads + at.sums;
  }
  by_type(params->dtype, D, [&](auto tag) {
    typedef typename decltype(tag)::type T;
    constexpr int VEC = decltype(tag)::vec;
    const Positions<T> positions{static_cast<T*>(dP),
                                 parts > 1 ? static_cast<float*>(params->workspace) + (at.words - at.positions) : nullptr,
                                 static_cast<size_t>(N) * D,
                                 static_cast<size_t>(params->position_offset) * D,
                                 static_cast<size_t>(params->positions) * D,
                                 static_cast<uint32_t>(B), lanes, parts, columns};
    const dim3 grid(table_blocks + static_cast<uint32_t>(position_blocks), (D / VEC + rows.lanes - 1) / rows.lanes);
    if (direct) {
      const auto kernel = n <= kFewTokens ? direct_kernel<T, VEC, kFewTokens> : direct_kernel<T, VEC, kDirectTokens>;
      kernel<<<grid, dim3(kSumThreads), 0, s>>>(
          Ids{ids, params->id_bytes == 8, V, params->padding_idx}, rows, static_cast<const T*>(dE), static_cast<T*>(dW), of_rows,
          table_blocks, positions);
    } else {
      sum_kernel<T, VEC><<<grid, dim3(kSumThreads), 0, s>>>(rows, static_cast<const T*>(dE), static_cast<T*>(dW), positions,
                                                            table_blocks);
    }
    if (parts > 1)
      join_positions_kernel<T><<<dim3(static_cast<uint32_t>((positions.width + 63) / 64)), dim3(kSumThreads), 0, s>>>(positions);
    if (dW != nullptr && !direct) {
      const dim3 join((at.units + kJoinWaves - 1) / kJoinWaves);
      if (D % 4 == 0) join_kernel<T, 4><<<join, dim3(64 * kJoinWaves), 0, s>>>(rows, static_cast<T*>(dW));
      else join_kernel<T, 1><<<join, dim3(64 * kJoinWaves), 0, s>>>(rows, static_cast<T*>(dW));
    }
  });
  if (err == hipSuccess) err = hipGetLastError();
  return err == hipSuccess ? COTTEN_OK : COTTEN_ERR_LAUNCH;
}

}  // extern "C"
