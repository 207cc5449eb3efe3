// drop.h -- the generator of dropout (formulas in fewbit_residual.h).
//
// Eight elements share a block of four words, so that eight elements of a lane need one run of
// the generator.  A round is two products of 32 by 32 bits, which
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

// A wave's 512 consecutive elements, eight to a lane, by accesses of 16 bytes that lie next to
// each other (two of 32-bit elements 1 KB apart: 32 bytes of a lane at a time would bring
// every line twice; 32768 x 1024 elements through dropout 56 us, so 43): element i of lane l
// is 8 l + i of 16-bit elements, and 4 l + i, 256 + 4 l + i - 4 of 32-bit ones.
constexpr int kWaveElements = kWave * 8;
template <class T>
struct Chunk {
  static constexpr int kAccesses = sizeof(T) / 2, kEach = 8 / kAccesses;

  // `first`: the wave's first element, relative to the stream
  template <int P>
  __device__ __forceinline__ static void load(const Stream& s, uint32_t first, int lane, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < kAccesses; ++j) {
      float v[kEach];
      s.template load<T, P>(first * sizeof(T) + j * 1024 + lane * 16, v);
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[j * kEach + i] = v[i];
    }
  }
  template <int P>
  __device__ __forceinline__ static void store(const Stream& s, uint32_t first, int lane, const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < kAccesses; ++j) {
      float v[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) v[i] = x[j * kEach + i];
      s.template store<T, P>(first * sizeof(T) + j * 1024 + lane * 16, v);
    }
  }
  // The same elements of a tensor of floats, and of bytes (packed in two words).
  template <int P>
  __device__ __forceinline__ static void store_floats(const Stream& s, uint32_t first, int lane, const float (&x)[8]) {
    if constexpr (kAccesses == 2)
      store<P>(s, first, lane, x);
    else
      s.template store<float, P>(first * 4 + lane * 32, x);
  }
  template <int P>
  __device__ __forceinline__ static void store_bytes(const Stream& s, uint32_t first, int lane, u32x2 x) {
    if constexpr (kAccesses == 2) {
      s.template put<P>(first + lane * 4, static_cast<uint32_t>(x[0]));
      s.template put<P>(first + 256 + lane * 4, static_cast<uint32_t>(x[1]));
    } else {
      s.template put<P>(first + lane * 8, x);
    }
  }
};

// A kept element.  The product passes an empty register barrier where it may be stored in fp16:
// the compiler would round it straight to that, and the result would not be that of fp32.
template <class T>
__device__ __forceinline__ float scaled(float x, const Drop& d) {
  x *= d.scale;
  if constexpr (__is_same(T, _Float16)) asm("" : "+v"(x));
  return x;
}

// A lane's elements of the 512 from 8 * block on.  Of 32-bit elements two lanes share a block
// in each access: the even one runs the generator for the first, the odd one for the second,
// and they hand each other the other's half.
template <class T>
__device__ __forceinline__ void drop(const Drop& d, Key key, uint64_t block, int lane, float (&x)[8]) {
  uint32_t c[4];
  if constexpr (Chunk<T>::kAccesses == 1) {
    words(block + lane, key, d.site, c);
  } else {
    const bool odd = lane % 2;
    uint32_t own[4];
    words(block + lane / 2 + (odd ? 32 : 0), key, d.site, own);
    uint32_t got[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      got[i] = __builtin_bit_cast(uint32_t, dpp<0xb1 /* quad_perm 1,0,3,2 */>(__builtin_bit_cast(float, odd ? own[i] : own[2 + i])));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[i] = odd ? got[i] : own[i];
      c[2 + i] = odd ? own[2 + i] : got[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = i % 2 ? c[i / 2] >> 16 : c[i / 2] & 0xFFFFu;
    x[i] = u >= d.border ? scaled<T>(x[i], d) : 0.0f;
  }
}

}  // namespace block
