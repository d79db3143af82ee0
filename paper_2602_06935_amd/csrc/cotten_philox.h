// The counter-based generator of the dropout: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011).  Elements are numbered through a tensor; eight of them share a counter, (number / 8,
// offset), under the seed as the key, and take 16 of its 128 bits each, in order.  An element whose 16 bits are below
// `out_of` is dropped, so p is a multiple of 2^-16, and the factor of what is kept is exact for that p.  (32 bits an element
// would be twice the rounds: the products of two words take four times as long as other operations.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cotten {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

struct Drop {
  uint64_t seed, offset;
  const long long* step;  // added to offset, or nullptr
  uint32_t out_of;        // of 65536; 0: nothing is dropped
  float factor;
};

// Where a kernel's generator stands: read once.
struct Lots {
  uint32_t k0, k1, c2, c3, out_of;
  float factor;
  __device__ __forceinline__ explicit Lots(const Drop& d) {
    const uint64_t offset = d.offset + (d.step == nullptr ? 0ull : static_cast<uint64_t>(*d.step));
    k0 = static_cast<uint32_t>(d.seed);
    k1 = static_cast<uint32_t>(d.seed >> 32);
    c2 = static_cast<uint32_t>(offset);
    c3 = static_cast<uint32_t>(offset >> 32);
    out_of = d.out_of;
    factor = d.factor;
  }
  __device__ __forceinline__ u32x4_t draw(uint64_t group) const {
    u32x4_t x = {static_cast<uint32_t>(group), static_cast<uint32_t>(group >> 32), c2, c3};
    uint32_t a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t first = static_cast<uint64_t>(x[0]) * 0xD2511F53u, second = static_cast<uint64_t>(x[2]) * 0xCD9E8D57u;
      x = u32x4_t{static_cast<uint32_t>(second >> 32) ^ x[1] ^ a, static_cast<uint32_t>(second),
                  static_cast<uint32_t>(first >> 32) ^ x[3] ^ b, static_cast<uint32_t>(first)};
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    return x;
  }
  // The 16 bits of eight elements from number `at` on, two to a word.  ALIGNED: `at` is a multiple of eight; otherwise they
  // come from two counters.
  template <bool ALIGNED>
  __device__ __forceinline__ u32x4_t of(uint64_t at) const {
    u32x4_t w = draw(at >> 3);
    if constexpr (!ALIGNED) {
      const uint32_t skip = static_cast<uint32_t>(at) & 7u;
      const u32x4_t v = draw((at >> 3) + 1);
      uint32_t x[8] = {w[0], w[1], w[2], w[3], v[0], v[1], v[2], v[3]};
#pragma unroll
      for (int i = 0; i < 6; ++i) x[i] = (skip & 4u) ? x[i + 2] : x[i];
#pragma unroll
      for (int i = 0; i < 5; ++i) x[i] = (skip & 2u) ? x[i + 1] : x[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (skip & 1u) ? (x[i] >> 16) | (x[i + 1] << 16) : x[i];
    }
    return w;
  }
  __device__ __forceinline__ bool keeps(const u32x4_t& w, int i) const {
    return ((i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu) >= out_of;
  }
};

}  // namespace cotten
