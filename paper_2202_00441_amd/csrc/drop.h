// drop.h -- the generator of dropout (formulas in fewbit_residual.h).
//
// Eight elements share a block of four words, so that an access of 16 bytes of 16-bit
// elements needs one run of the generator.  A round is two products of 32 by 32 bits, which
// the vector units form in one instruction each, and four exclusive ors.
#pragma once

#include <cmath>

#include "block.h"
#include "fewbit_residual.h"

namespace block {

struct Drop {
  const int64_t* at;        // the seed's place on the device, or NULL
  uint32_t k0, k1, site;
  uint32_t border;          // t
  float scale;              // 65536 / (65536 - t)
};

// A status, or what the kernels take.
inline int drop_of(const fewbit_drop& d, Drop& r) {
  if (!(d.p >= 0.0 && d.p <= 1.0) || d.reserved != 0) return FEWBIT_E_INVALID;
  if (reinterpret_cast<uintptr_t>(d.seed_at) % 8 != 0) return FEWBIT_E_ALIGN;
  r.at = d.seed_at;
  r.k0 = static_cast<uint32_t>(d.seed);
  r.k1 = static_cast<uint32_t>(static_cast<uint64_t>(d.seed) >> 32);
  r.site = d.site;
  r.border = static_cast<uint32_t>(std::nearbyint(d.p * 65536.0));
  r.scale = r.border < 65536 ? static_cast<float>(65536.0 / (65536 - r.border)) : 0.0f;
  return FEWBIT_OK;
}

struct Key {
  uint32_t k0, k1;
};
__device__ __forceinline__ Key key_of(const Drop& d) {
  if (!d.at) return {d.k0, d.k1};
  const uint64_t seed = static_cast<uint64_t>(*d.at);
  return {static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(seed))),
          static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(seed >> 32)))};
}

// The four words of a block.
__device__ __forceinline__ void words(uint64_t block, Key key, uint32_t site, uint32_t (&c)[4]) {
  c[0] = static_cast<uint32_t>(block);
  c[1] = static_cast<uint32_t>(block >> 32);
  c[2] = site;
  c[3] = 0;
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    const uint64_t a = uint64_t{0xD2511F53u} * c[0], b = uint64_t{0xCD9E8D57u} * c[2];
    const uint32_t k0 = key.k0 + i * 0x9E3779B9u, k1 = key.k1 + i * 0xBB67AE85u;
    c[0] = static_cast<uint32_t>(b >> 32) ^ c[1] ^ k0;
    c[1] = static_cast<uint32_t>(b);
    c[2] = static_cast<uint32_t>(a >> 32) ^ c[3] ^ k1;
    c[3] = static_cast<uint32_t>(a);
  }
}

// Element i of eight is kept.
__device__ __forceinline__ bool kept(const uint32_t (&c)[4], int i, uint32_t border) {
  const uint32_t u = i % 2 ? c[i / 2] >> 16 : c[i / 2] & 0xFFFFu;
  return u >= border;
}

// Eight elements from 8 * block on.
__device__ __forceinline__ void drop(const Drop& d, Key key, uint64_t block, float (&x)[8]) {
  uint32_t c[4];
  words(block, key, d.site, c);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = kept(c, i, d.border) ? x[i] * d.scale : 0.0f;
}

}  // namespace block
