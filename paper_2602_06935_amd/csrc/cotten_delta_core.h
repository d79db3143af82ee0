// Device code shared by the kernels of the gated delta rule: the pieces that matrix-core operands are cut into, row
// loads in the layout of the products, and what a chunk of 32 tokens needs before its state is known.
//
// The operation, for a slice (b,h) with unit rows k^ = k / sqrt(|k|^2 + eps), q^ likewise, a_t = exp(g_t):
//
//     u_t = beta_t (v_t - a_t S_{t-1}^T k^_t)      S_t = a_t S_{t-1} + k^_t u_t^T      o_t = scale * S_t^T q^_t
//
// (a masked token: a = 1, beta = 0).  Over a chunk, with S the state before it, G the inclusive sums of g inside it and
// everything row by row:
//
//     N_ij = e^(G_i - G_j) k^_i . k^_j  (j < i)     T = (I + diag(beta) N)^-1
//     U = T beta (V - e^G (K^ S))                   O = scale (e^G (Q^ S) + M U),  M_ij = e^(G_i - G_j) q^_i . k^_j (j <= i)
//     S' = e^(G_C) S + K^^T (e^(G_C - G) U)
//
// T and M do not depend on the state: "producer" waves make them, ahead of the waves that carry the state along.
//
// Precision.  States and gate gradients leave in fp32, and an error of u is written into the state, so nothing is
// rounded to 16 bits on the way: an operand is cut into bf16 pieces, x = h + m + l exactly (fp32: three pieces; fp16: two;
// bf16: itself), and a product is the sum of the products of pieces that reach 24 bits (the norms 1 / r(x) and the
// decays are factors of the results, so raw 16-bit rows stay exact operands).  For bf16 rows a product with the state
// is three matrix instructions, for fp32 rows six, a fifth and 2/5 of what fp32 matrix instructions would take.
// Sums of g are fp64: differences of sums that a strong decay has made large would lose the weak decays after it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cotten {
namespace delta {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

constexpr int kChunk = 32;                       // tokens of a chunk: the depth of one matrix instruction
constexpr uint32_t kNowhere = 0x80000000u;       // a byte offset beyond every slice: such loads bring zeros

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

// A barrier for what waves pass each other through LDS: loads and stores of global memory stay on their way across it
// (a full barrier waits for them, and nothing that a producer had asked for a chunk ahead would come early).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ f32x4_t mfma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma(float a, float b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// ---- pieces ----------------------------------------------------------------------------------------------------

template <int P>
struct Pieces {
  bf16x8_t p[P];  // p[0] the leading bits
};

// Eight values as three pieces of eight significant bits each, exactly: h the upper half of the word, m of what is left, l
// the rest, which fits.  OTHER: how many pieces the operand has that they meet.  With one, every product is kept, and m is the upper
// half of what is left.  With more, the products of m and l with l are left out (see mul), and m is rounded: an m cut off leaves
// an l of x's sign, and products left out that add up (mean 0.69 and 1.0 rms of 2^-24 of a product; rounded 0 and 0.38).
// Conversions take longer than bit operations: all operands with m cut off / as they are / all rounded, 16 x 4 x 4096 x 64 bf16
// forward 126.4 / 128.6 / 135 us, 128 x 4 x 200 x 64 bf16 24.7 / 25.2 / 25.9, 64 x 2 x 197 x 128 fp16 29.2 / 30.2 / 30.4.  (Half a
// step of m added to its bits in place of the conversion: 129.0, 25.0 and 29.8, but fp32, where all are rounded, 256 x 2 x
// 200 x 32 21.5 for 21.0, 128 x 4 x 200 x 64 45.0 for 44.0.)
__device__ __forceinline__ float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint32_t uppers(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
template <int OTHER>
__device__ __forceinline__ Pieces<3> cut(const float (&x)[8]) {
  u32x4_t h, m, l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[2 * i], b = x[2 * i + 1], ra = a - upper(a), rb = b - upper(b);
    h[i] = uppers(a, b);
    if constexpr (OTHER > 1) {
      bf16x2_t v;
      v[0] = static_cast<__bf16>(ra);
      v[1] = static_cast<__bf16>(rb);
      uint32_t w = __builtin_bit_cast(uint32_t, v);
      asm("" : "+v"(w));  // (both halves from the one conversion: the compiler would make the lower one again)
      m[i] = w;
      l[i] = uppers(ra - __uint_as_float(w << 16), rb - upper(__uint_as_float(w)));
    } else {
      m[i] = uppers(ra, rb);
      l[i] = uppers(ra - upper(ra), rb - upper(rb));
    }
  }
  Pieces<3> r;
  r.p[0] = __builtin_bit_cast(bf16x8_t, h);
  r.p[1] = __builtin_bit_cast(bf16x8_t, m);
  r.p[2] = __builtin_bit_cast(bf16x8_t, l);
  return r;
}
template <int OTHER>
__device__ __forceinline__ Pieces<3> cut(f32x4_t a, f32x4_t b) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return cut<OTHER>(x);
}

// The pieces that values of E's are made of (fewer than three where they are 16-bit values: nothing is left for l).
template <class E>
__device__ __forceinline__ Pieces<E::kPieces> cut_elements(f32x4_t a, f32x4_t b) {
  const Pieces<3> c = cut<E::kPieces == 3 ? 3 : 1>(a, b);
  Pieces<E::kPieces> r;
#pragma unroll
  for (int i = 0; i < E::kPieces; ++i) r.p[i] = c.p[i];
  return r;
}

// c += A B, the products of pieces that reach 24 bits, the small ones first.  (Of two operands in three pieces, m l is left
// out: with rounded m 0.38 rms of 2^-24 of a product, 2^-22 at most, of either sign.)
template <int PA, int PB>
__device__ __forceinline__ f32x4_t mul(const Pieces<PA>& a, const Pieces<PB>& b, f32x4_t c) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i)
      if (s - i >= 0 && s - i < PB) c = mfma(a.p[i], b.p[s - i], c);
  return c;
}

// N products side by side: no matrix instruction waits for the one before it.
template <int N, int PA, int PB>
__device__ __forceinline__ void mul_left(const Pieces<PA> (&a)[N], const Pieces<PB>& b, f32x4_t (&c)[N]) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (s - i >= 0 && s - i < PB) c[n] = mfma(a[n].p[i], b.p[s - i], c[n]);
}
template <int N, int PA, int PB>
__device__ __forceinline__ void mul_right(const Pieces<PA>& a, const Pieces<PB> (&b)[N], f32x4_t (&c)[N]) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (s - i >= 0 && s - i < PB) c[n] = mfma(a.p[i], b[n].p[s - i], c[n]);
}

// ---- element formats: eight consecutive elements of a row ---------------------------------------------------------

struct F32 {
  static constexpr int kBytes = 4, kPieces = 3;
  struct Raw {
    u32x4_t a, b;
  };
  static __device__ __forceinline__ Raw load(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return Raw{__builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0),
               __builtin_amdgcn_raw_buffer_load_b128(r, off + 16, 0, 0)};
  }
  static __device__ __forceinline__ void unpack(const Raw& w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __uint_as_float(w.a[i]);
      x[4 + i] = __uint_as_float(w.b[i]);
    }
  }
  static __device__ __forceinline__ Pieces<3> pieces(const Raw& w) {
    float x[8];
    unpack(w, x);
    return cut<3>(x);
  }
  typedef uint32_t One;  // an element as it was loaded: turned into a float where it is used, not where it would be waited for
  static __device__ __forceinline__ One load_one(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0);
  }
  static __device__ __forceinline__ float value(One w) { return __uint_as_float(w); }
  static __device__ __forceinline__ f32x4_t load_four(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
  }
  static __device__ __forceinline__ void store_one(__amdgpu_buffer_rsrc_t r, uint32_t off, float x) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), r, off, 0, 0);
  }
  static __device__ __forceinline__ void store_four(__amdgpu_buffer_rsrc_t r, uint32_t off, f32x4_t x) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), r, off, 0, 0);
  }
};

template <class T>
struct Half {
  static constexpr int kBytes = 2;
  typedef u32x4_t Raw;
  static __device__ __forceinline__ Raw load(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
  }
  static __device__ __forceinline__ float value(uint16_t bits) { return static_cast<float>(__builtin_bit_cast(T, bits)); }
  static __device__ __forceinline__ uint16_t bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<T>(x)); }
  static __device__ __forceinline__ void unpack(const Raw& w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = value(static_cast<uint16_t>(w[i] & 0xffffu));
      x[2 * i + 1] = value(static_cast<uint16_t>(w[i] >> 16));
    }
  }
  typedef uint32_t One;  // (a 16-bit variable would be masked, and waited for, where it is loaded)
  static __device__ __forceinline__ One load_one(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0));
  }
  static __device__ __forceinline__ float value(One w) { return value(static_cast<uint16_t>(w)); }
  static __device__ __forceinline__ f32x4_t load_four(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    const u32x2_t w = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
    return f32x4_t{value(w[0]), value(w[0] >> 16), value(w[1]), value(w[1] >> 16)};
  }
  static __device__ __forceinline__ void store_one(__amdgpu_buffer_rsrc_t r, uint32_t off, float x) {
    __builtin_amdgcn_raw_buffer_store_b16(bits(x), r, off, 0, 0);
  }
  static __device__ __forceinline__ void store_four(__amdgpu_buffer_rsrc_t r, uint32_t off, f32x4_t x) {
    typedef T quad __attribute__((ext_vector_type(4)));  // (two conversions of pairs; of one value each they would be four, and packed)
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2_t, __builtin_convertvector(x, quad)), r, off, 0, 0);
  }
};
struct Bf16 : Half<__bf16> {
  static constexpr int kPieces = 1;
  static __device__ __forceinline__ Pieces<1> pieces(const Raw& w) {
    Pieces<1> r;
    r.p[0] = __builtin_bit_cast(bf16x8_t, w);
    return r;
  }
};
struct F16 : Half<_Float16> {  // 11 significant bits: two pieces
  static constexpr int kPieces = 2;
  static __device__ __forceinline__ Pieces<2> pieces(const Raw& w) {
    float x[8];
    unpack(w, x);
    const Pieces<3> c = cut<1>(x);
    Pieces<2> r;
    r.p[0] = c.p[0];
    r.p[1] = c.p[1];
    return r;
  }
};

// ---- arguments --------------------------------------------------------------------------------------------------

struct Args {
  const unsigned char* Q;
  const unsigned char* K;
  const unsigned char* V;
  const unsigned char* dO;
  const float* g;
  const float* beta;
  const uint8_t* mask;          // [B,N] or nullptr
  unsigned char* O;             // nullptr: states only
  unsigned char* dQ;
  unsigned char* dK;
  unsigned char* dV;
  float* dg;
  float* dbeta;
  const float* initial_state;   // [B*H][D][D] or nullptr
  float* final_state;
  const float* dfinal_state;
  float* dinitial_state;
  float* states;                // [slice][chunk][D][D]: the state before every chunk, or nullptr
  float* rows_u;                // [slice][chunk * 32][D]: U, or nullptr
  float* dstates;               // [slice][chunk][D][D]: the gradient of the state after every chunk (backward)
  float* rows_z;                // [slice][chunk * 32][D]: Z (backward)
  // Sequences cut into segments (see segments_of): what a segment makes of the state before it, S -> M S + R, and the
  // gradient of the state before it where that of the state after it is zero.
  float* transitions;           // [slice][segment][2][D][D]: R, M
  float* carries;               // [slice][segment][D][D] (backward)
  int segments, segment_chunks;
  int H, N, chunks;
  long long stride_batch, stride_head;  // of the tensors, in bytes
  uint32_t stride_row;
  long long gate_batch, gate_head;      // of g and beta, in elements
  int gate_row;
  float scale, eps;
};

// A buffer of `bytes` from `base`, which are the same in all lanes: kept in scalar registers (left to itself the compiler
// has put descriptors made inside a loop into vector registers, and a loop over lanes around every load).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(p)), hi = __builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((static_cast<uint64_t>(hi) << 32) | lo), 0,
                                           __builtin_amdgcn_readfirstlane(static_cast<int>(bytes)), 0x00020000);
}

// What a wave knows of its slice.
struct Slice {
  long long rows;       // byte offset of row 0 in Q, K, V, O ...
  long long gates;      // element offset of token 0 in g, beta ...
  const uint8_t* mask;  // of the sequence, or nullptr
  uint32_t bytes;       // from row 0 to the end of row N-1
  __device__ __forceinline__ Slice(const Args& a, int slice, uint32_t row_bytes) {
    const int b = slice / a.H, h = slice - b * a.H;
    rows = b * a.stride_batch + h * a.stride_head;
    gates = b * a.gate_batch + h * a.gate_head;
    mask = a.mask == nullptr ? nullptr : a.mask + static_cast<long long>(b) * a.N;
    bytes = static_cast<uint32_t>(a.N - 1) * a.stride_row + row_bytes;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t of(const unsigned char* base) const {
    return buffer(base + rows, bytes);
  }
  // from a chunk's first row on: a lane's offsets are the same in every chunk, and rows beyond the sequence are beyond the
  // buffer (loads bring zeros, stores are dropped)
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t of(const unsigned char* base, int chunk, uint32_t stride) const {
    const uint32_t skip = static_cast<uint32_t>(kChunk * chunk) * stride;
    return buffer(base + rows + skip, skip < bytes ? bytes - skip : 0);
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t of_gate(const Args& a, const float* base) const {
    return buffer(base + gates, ((a.N - 1) * a.gate_row + 1) * 4);
  }
};

// The tokens of a chunk that take part.  A byte of the mask is asked for a chunk ahead of the rows that hang on it.
struct Live {
  __amdgpu_buffer_rsrc_t mask;
  bool all;
  int N;
  __device__ __forceinline__ Live(const Args& a, const Slice& s)
      : mask(buffer(s.mask, s.mask == nullptr ? 0 : a.N)),
        all(s.mask == nullptr),
        N(a.N) {}
  // of token 32 * chunk + lane%32 (beyond the sequence: 0)
  __device__ __forceinline__ uint32_t fetch(int chunk, int lane) const {
    return __builtin_amdgcn_raw_buffer_load_b8(mask, static_cast<uint32_t>(kChunk * chunk + (lane & 31)), 0, 0);
  }
  // bit t: token 32 * chunk + t takes part
  __device__ __forceinline__ uint32_t bits(uint32_t byte, int chunk) const;
};

// Bit t: token 32 * chunk + t exists.
__device__ __forceinline__ uint32_t existing(int N, int chunk) {
  const int left = N - kChunk * chunk;
  return left >= kChunk ? ~0u : (1u << left) - 1u;
}

__device__ __forceinline__ uint32_t Live::bits(uint32_t byte, int chunk) const {
  return all ? existing(N, chunk) : static_cast<uint32_t>(__ballot(byte != 0));
}
// A gate of token 32 * chunk + lane%32; 0 where it takes no part.
__device__ __forceinline__ uint32_t fetch_gate(const Args& a, __amdgpu_buffer_rsrc_t r, int chunk, uint32_t live, int lane) {
  const uint32_t off = static_cast<uint32_t>(kChunk * chunk + (lane & 31)) * a.gate_row * 4;
  return __builtin_amdgcn_raw_buffer_load_b32(r, ((live >> (lane & 31)) & 1u) ? off : kNowhere, 0, 0);
}

// An offset, or one beyond every buffer where the token of the chunk takes no part.
__device__ __forceinline__ uint32_t offset_if(uint32_t live, int token, uint32_t off) { return ((~live >> token) << 31) | off; }

// ---- decays -----------------------------------------------------------------------------------------------------

// A sum of g * log2(e) as two floats.  Their differences are formed part by part: what rounding is left costs
// 2^x |x| 2^-24 at most, which for decays is less than a rounding of 1, the largest of the factors it is summed with.
struct Sum {
  float hi, lo;
};
__device__ __forceinline__ Sum split(double x) {
  const float hi = static_cast<float>(x);
  return Sum{hi, static_cast<float>(x - hi)};
}
// 2^(a - b)
__device__ __forceinline__ float pow2(Sum a, Sum b) { return __builtin_amdgcn_exp2f((a.hi - b.hi) + (a.lo - b.lo)); }
__device__ __forceinline__ float pow2(Sum a) { return __builtin_amdgcn_exp2f(a.hi + a.lo); }
__device__ __forceinline__ Sum of_lane(Sum x, int lane) { return Sum{__shfl(x.hi, lane), __shfl(x.lo, lane)}; }

// The lanes of a row of 16 shifted right by N (lanes without a source: 0).
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double move_lanes(double x) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(w), CTRL, ROWS, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(w >> 32), CTRL, ROWS, 0xF, true);
  return __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
}

// Inclusive sums of g * log2(e) over the chunk's 32 tokens, the same in both halves of the wave (lane & 31 is the token).
// A decay to nothing (g = -inf) counts as 2^-100000: fp32 knows no difference, and later differences stay numbers.
__device__ __forceinline__ Sum scan_decays(float g, int lane) {
  double x = static_cast<double>(g) * 1.4426950408889634;
  x = x < -100000.0 ? -100000.0 : x;
  x += move_lanes<0x111>(x);  // row_shr 1, 2, 4, 8: sums inside rows of 16
  x += move_lanes<0x112>(x);
  x += move_lanes<0x114>(x);
  x += move_lanes<0x118>(x);
  const double first = move_lanes<0x15F>(x);  // the last lane of every row, to all of its lanes
  const uint64_t w = __builtin_bit_cast(uint64_t, first);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(w), 0), hi = __builtin_amdgcn_readlane(static_cast<int>(w >> 32), 0);
  const double row0 = __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
  return split((lane & 16) ? x + row0 : x);
}
// ... of the whole chunk
__device__ __forceinline__ Sum last_of_scan(Sum x) {
  return Sum{__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x.hi), 31)),
             __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x.lo), 31))};
}

// Inclusive sums over the chunk's tokens (lane & 31) of the lower half of a wave: of those up to the lane's, and from it on.
template <int CTRL>
__device__ __forceinline__ float add_moved(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float of_fixed_lane(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(x)), lane));
}
__device__ __forceinline__ float sums_up_to(float x, int lane) {
  x = add_moved<0x118>(add_moved<0x114>(add_moved<0x112>(add_moved<0x111>(x))));  // row_shr 1, 2, 4, 8
  const float row0 = of_fixed_lane(x, 15);
  return (lane & 16) ? x + row0 : x;
}
__device__ __forceinline__ float sums_from(float x, int lane) {
  x = add_moved<0x108>(add_moved<0x104>(add_moved<0x102>(add_moved<0x101>(x))));  // row_shl 1, 2, 4, 8
  const float row1 = of_fixed_lane(x, 16);
  return (lane & 16) ? x : x + row1;
}
// Sum over the 16 lanes of a row, in its last lane.
__device__ __forceinline__ float sum_of_row(float x) {
  return add_moved<0x118>(add_moved<0x114>(add_moved<0x112>(add_moved<0x111>(x))));
}

// Sum over the four lanes with the same lane % 16.
__device__ __forceinline__ float over_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ---- rows in LDS ------------------------------------------------------------------------------------------------
//
// 32 rows of a chunk, a plane per piece.  A lane of a product holds, of a block of 32 columns, the columns 4g .. 4g+3
// and 16+4g .. 16+4g+3 (g = lane / 16): the rows of two 16-row result tiles that it holds, so a result is fed back as an
// operand without moving between lanes.  Rows are kept in that order ("slots"): the operand is one 16-byte read.
// Writes of loaded rows and the reads of columns take 8 of every 16 bytes, which is half of the banks: 28 % of the active LDS
// cycles of the forward are conflicts, 31 % of the adjoint walk's and 33 % of the gradient kernel's (128 x 4 x 200 x 64 bf16).

template <int D, int P>
struct Rows {
  static constexpr int kWidth = D < 32 ? 32 : D;          // (narrow rows are followed by zeros)
  static constexpr int kBlocks = kWidth / 32;
  static constexpr int kStride = kWidth * 2 + 16;         // bytes; the padding spreads the 16-byte reads of rows over the banks
  static constexpr int kPlane = kChunk * kStride;
  static constexpr int kBytes = P * kPlane;

  // columns 32 kb + 8 g .. + 7 of a row, as loads in natural order bring them
  static __device__ __forceinline__ void put(unsigned char* at, int row, int kb, int g, const Pieces<P>& x) {
    const int slot = (g & 1) * 32 + (g >> 1) * 8;  // bytes: columns 8g .. 8g+3 (8g+4 .. +7: 16 bytes on)
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const u32x4_t w = __builtin_bit_cast(u32x4_t, x.p[i]);
      unsigned char* p = at + i * kPlane + row * kStride + kb * 64 + slot;
      *reinterpret_cast<u32x2_t*>(p) = u32x2_t{w[0], w[1]};
      *reinterpret_cast<u32x2_t*>(p + 16) = u32x2_t{w[2], w[3]};
    }
  }
  // operand: row 16 tt + lane%16, depth = the columns of block kb
  static __device__ __forceinline__ Pieces<P> row_operand(const unsigned char* at, int tt, int kb, int lane) {
    Pieces<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i)
      r.p[i] = *reinterpret_cast<const bf16x8_t*>(at + i * kPlane + (16 * tt + (lane & 15)) * kStride + kb * 64 + (lane >> 4) * 16);
    return r;
  }
  // operand: column 16 dt + lane%16, depth = the 32 tokens (in the slot order of a pair of result tiles)
  static __device__ __forceinline__ Pieces<P> column_operand(const unsigned char* at, int dt, int lane) {
    typedef bf16x4_t __attribute__((address_space(3))) * lds_v4;
    const int s = lane & 15, g = lane >> 4;
    const unsigned char* p = at + (4 * g + (s >> 2)) * kStride + (dt >> 1) * 64 + (s & 3) * 16 + (dt & 1) * 8;
    Pieces<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(p + i * kPlane));
      const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(p + i * kPlane + 16 * kStride));
      r.p[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    return r;
  }
};

// A 32 x 32 triangular operand in LDS in the order the products read it: [tile][piece][lane] 16 bytes.
constexpr int kTriangleBytes = 2 * 3 * 64 * 16;
template <int OTHER>
__device__ __forceinline__ void put_triangle(unsigned char* at, int tile, int lane, f32x4_t lo, f32x4_t hi) {
  const Pieces<3> x = cut<OTHER>(lo, hi);
#pragma unroll
  for (int i = 0; i < 3; ++i) *reinterpret_cast<bf16x8_t*>(at + ((tile * 3 + i) * 64 + lane) * 16) = x.p[i];
}
__device__ __forceinline__ Pieces<3> triangle_operand(const unsigned char* at, int tile, int lane) {
  Pieces<3> r;
#pragma unroll
  for (int i = 0; i < 3; ++i) r.p[i] = *reinterpret_cast<const bf16x8_t*>(at + ((tile * 3 + i) * 64 + lane) * 16);
  return r;
}

// ---- what the producers read and make -----------------------------------------------------------------------------

// The 32 rows of a chunk of Q or K straight in the layout of the products (columns in natural order).
template <class E, int D>
struct RowTile {
  static constexpr int kBlocks = Rows<D, E::kPieces>::kBlocks;
  typename E::Raw raw[2][kBlocks];
  // r: from the chunk's first row on
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t stride, uint32_t live, int lane) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int row = 16 * tt + (lane & 15);
      const uint32_t off = static_cast<uint32_t>(row) * stride + (lane >> 4) * 8 * E::kBytes;
      const uint32_t at = offset_if(live, row, D >= 32 || (lane >> 4) * 8 < D ? off : kNowhere);
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb) raw[tt][kb] = E::load(r, at + kb * 32 * E::kBytes);
    }
  }
  __device__ __forceinline__ Pieces<E::kPieces> operand(int tt, int kb) const { return E::pieces(raw[tt][kb]); }
  __device__ __forceinline__ void put(unsigned char* at, int lane) const {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int kb = 0; kb < kBlocks; ++kb)
        Rows<D, E::kPieces>::put(at, 16 * tt + (lane & 15), kb, lane >> 4, operand(tt, kb));
  }
};

// Result rows 4g .. 4g+3 = rows of X tile `a`, result column lane%16 = row of Y tile `b`: X_a Y_b^T.
template <class E, int D>
__device__ __forceinline__ f32x4_t dots(const RowTile<E, D>& X, int a, const RowTile<E, D>& Y, int b) {
  f32x4_t c = {0, 0, 0, 0};
#pragma unroll
  for (int kb = 0; kb < RowTile<E, D>::kBlocks; ++kb) c = mul(X.operand(a, kb), Y.operand(b, kb), c);
  return c;
}

// 1 / sqrt(square + eps) of row 16 tt + lane%16, the same in the four lanes that share it, from the products of the tile's
// rows with one another, whose diagonal are the squares; 0 for a row that was not loaded (whatever eps is: its products
// are zeros and stay zeros).
__device__ __forceinline__ float inverse_norm(f32x4_t products, int tt, float eps, uint32_t live, int lane) {
  const int c = lane & 15;
  const float x = (c & 2) ? ((c & 1) ? products[3] : products[2]) : ((c & 1) ? products[1] : products[0]);
  const float square = over_groups((c >> 2) == (lane >> 4) ? x : 0.0f);
  return ((live >> (16 * tt + c)) & 1u) ? __builtin_amdgcn_rsqf(square + eps) : 0.0f;
}

// A producer's own notes of a chunk, by token: sums of decays, and the factor of the row in the products it makes.
struct Notes {
  float hi[kChunk], lo[kChunk];
  float factor[kChunk];
  float other[kChunk];  // (keys, backward: the factor without beta)
};
// ... of the rows 4g .. 4g+3 of both halves, and of row lane%16
struct Noted {
  f32x4_t hi[2], lo[2], factor[2];
  Sum Gc[2];
  __device__ __forceinline__ Noted(const Notes& n, int lane) {
    const int c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      Gc[t] = Sum{n.hi[16 * t + c], n.lo[16 * t + c]};
      hi[t] = *reinterpret_cast<const f32x4_t*>(&n.hi[16 * t + 4 * g]);
      lo[t] = *reinterpret_cast<const f32x4_t*>(&n.lo[16 * t + 4 * g]);
      factor[t] = *reinterpret_cast<const f32x4_t*>(&n.factor[16 * t + 4 * g]);
    }
  }
  __device__ __forceinline__ Sum G(int t, int r) const { return Sum{hi[t][r], lo[t][r]}; }
};

constexpr int kSquareStride = 20;                    // floats per row of a 16 x 16 square (80 bytes: free of conflicts)
constexpr int kSquare = 16 * kSquareStride;
struct Scratch {  // of the wave that solves
  Notes notes;
  float a[2][kSquare];  // diagonal blocks of diag(beta) N, transposed
  float t[2][kSquare];  // diagonal blocks of T
};

// t_J = [i = J] - sum_{m > J} t_m A_mJ for J = 15 ... 0, in row i = lane%16; A: minus the column lane%16, so a term is one
// multiply-add with the value of lane J of each 16 lanes.  A row is one statement, and the two wait states between
// a register's last write and its use in other lanes are its first instruction: whatever the compiler puts before, a copy too.
#define COTTEN_TERM(M) "\n\tv_fmac_f32_dpp %[x], %[a" #M "], %[t" #M "] row_newbcast:%[j] row_mask:0xf bank_mask:0xf"
#define COTTEN_PAIR(M) [a##M] "v"(A[M]), [t##M] "v"(t[M])
#define COTTEN_TERMS_15 COTTEN_TERM(15)
#define COTTEN_TERMS_14 COTTEN_TERMS_15 COTTEN_TERM(14)
#define COTTEN_TERMS_13 COTTEN_TERMS_14 COTTEN_TERM(13)
#define COTTEN_TERMS_12 COTTEN_TERMS_13 COTTEN_TERM(12)
#define COTTEN_TERMS_11 COTTEN_TERMS_12 COTTEN_TERM(11)
#define COTTEN_TERMS_10 COTTEN_TERMS_11 COTTEN_TERM(10)
#define COTTEN_TERMS_9 COTTEN_TERMS_10 COTTEN_TERM(9)
#define COTTEN_TERMS_8 COTTEN_TERMS_9 COTTEN_TERM(8)
#define COTTEN_TERMS_7 COTTEN_TERMS_8 COTTEN_TERM(7)
#define COTTEN_TERMS_6 COTTEN_TERMS_7 COTTEN_TERM(6)
#define COTTEN_TERMS_5 COTTEN_TERMS_6 COTTEN_TERM(5)
#define COTTEN_TERMS_4 COTTEN_TERMS_5 COTTEN_TERM(4)
#define COTTEN_TERMS_3 COTTEN_TERMS_4 COTTEN_TERM(3)
#define COTTEN_TERMS_2 COTTEN_TERMS_3 COTTEN_TERM(2)
#define COTTEN_TERMS_1 COTTEN_TERMS_2 COTTEN_TERM(1)
#define COTTEN_PAIRS_15 COTTEN_PAIR(15)
#define COTTEN_PAIRS_14 COTTEN_PAIRS_15, COTTEN_PAIR(14)
#define COTTEN_PAIRS_13 COTTEN_PAIRS_14, COTTEN_PAIR(13)
#define COTTEN_PAIRS_12 COTTEN_PAIRS_13, COTTEN_PAIR(12)
#define COTTEN_PAIRS_11 COTTEN_PAIRS_12, COTTEN_PAIR(11)
#define COTTEN_PAIRS_10 COTTEN_PAIRS_11, COTTEN_PAIR(10)
#define COTTEN_PAIRS_9 COTTEN_PAIRS_10, COTTEN_PAIR(9)
#define COTTEN_PAIRS_8 COTTEN_PAIRS_9, COTTEN_PAIR(8)
#define COTTEN_PAIRS_7 COTTEN_PAIRS_8, COTTEN_PAIR(7)
#define COTTEN_PAIRS_6 COTTEN_PAIRS_7, COTTEN_PAIR(6)
#define COTTEN_PAIRS_5 COTTEN_PAIRS_6, COTTEN_PAIR(5)
#define COTTEN_PAIRS_4 COTTEN_PAIRS_5, COTTEN_PAIR(4)
#define COTTEN_PAIRS_3 COTTEN_PAIRS_4, COTTEN_PAIR(3)
#define COTTEN_PAIRS_2 COTTEN_PAIRS_3, COTTEN_PAIR(2)
#define COTTEN_PAIRS_1 COTTEN_PAIRS_2, COTTEN_PAIR(1)
#define COTTEN_ROW(J, M)                                                             \
  {                                                                                  \
    float x = i == J ? 1.0f : 0.0f;                                                  \
    asm("s_nop 1" COTTEN_TERMS_##M : [x] "+&v"(x) : COTTEN_PAIRS_##M, [j] "n"(J));   \
    t[J] = x;                                                                        \
  }
__device__ __forceinline__ void solve_rows(const float (&A)[16], float (&t)[16], int i) {
  t[15] = i == 15 ? 1.0f : 0.0f;
  COTTEN_ROW(14, 15)
  COTTEN_ROW(13, 14)
  COTTEN_ROW(12, 13)
  COTTEN_ROW(11, 12)
  COTTEN_ROW(10, 11)
  COTTEN_ROW(9, 10)
  COTTEN_ROW(8, 9)
  COTTEN_ROW(7, 8)
  COTTEN_ROW(6, 7)
  COTTEN_ROW(5, 6)
  COTTEN_ROW(4, 5)
  COTTEN_ROW(3, 4)
  COTTEN_ROW(2, 3)
  COTTEN_ROW(1, 2)
  COTTEN_ROW(0, 1)
}

// T = (I + A)^-1 for A = [[A0, 0], [A10, A1]], strictly lower: the diagonal blocks by substitution (as stable as solving
// token by token; powers of A would lose digits where keys repeat), and T10 = -T1 A10 T0.  `d0`, `d1`: A0 and A1 as
// results (row 4g + r, column lane%16).  In LDS afterwards: the rows of T0 and T1.
__device__ __forceinline__ void solve_blocks(Scratch* s, f32x4_t d0, f32x4_t d1, int lane) {
  const int c = lane & 15, g = lane >> 4;
  *reinterpret_cast<f32x4_t*>(&s->a[0][c * kSquareStride + 4 * g]) = d0;
  *reinterpret_cast<f32x4_t*>(&s->a[1][c * kSquareStride + 4 * g]) = d1;
  wave_fence();
  // row i = lane%16 of T of block (lane / 16) % 2: t_j = [i = j] - sum_{m > j} t_m A_mj.  Lane j has column j of A: what
  // all lanes need of it comes by a broadcast inside the 16 lanes.
  float A[16], t[16];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const f32x4_t w = *reinterpret_cast<const f32x4_t*>(&s->a[g & 1][c * kSquareStride + 4 * q]);
#pragma unroll
    for (int e = 0; e < 4; ++e) A[4 * q + e] = -w[e];
  }
  solve_rows(A, t, c);
#pragma unroll
  for (int q = 0; q < 4; ++q)  // (two lane groups write the same; a branch would keep the broadcasts out of the sums)
    *reinterpret_cast<f32x4_t*>(&s->t[g & 1][c * kSquareStride + 4 * q]) = f32x4_t{t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]};
  wave_fence();
}
__device__ __forceinline__ f32x4_t square_row(const float* m, int lane) {  // row lane%16, columns 4g .. 4g+3
  return *reinterpret_cast<const f32x4_t*>(&m[(lane & 15) * kSquareStride + 4 * (lane >> 4)]);
}
__device__ __forceinline__ f32x4_t square_column(const float* m, int lane) {  // column lane%16, rows 4g .. 4g+3
  f32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = m[(4 * (lane >> 4) + i) * kSquareStride + (lane & 15)];
  return r;
}
// A 16 x 16 product in fp32 over a depth of 16: lane holds row (column) lane%16 at depths 4g .. 4g+3
__device__ __forceinline__ f32x4_t square_product(f32x4_t a, f32x4_t b) {
  f32x4_t c = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = mfma(a[i], b[i], c);
  return c;
}

}  // namespace delta
}  // namespace cotten
