// block.h -- what the block operators' sources share: storage types, cross-lane
// steps inside a wave, launches and the host's checks.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../include/fewbit_block.h"

namespace block {

constexpr int kWave = 64;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- storage types
template <int DT>
struct Store;
template <>
struct Store<FEWBIT_F32> {
  using type = float;
};
template <>
struct Store<FEWBIT_F16> {
  using type = _Float16;
};
template <>
struct Store<FEWBIT_BF16> {
  using type = __bf16;
};

// N consecutive values as fp32, from and to an address with `N * size` (at most
// 16) bytes of alignment; conversion to 16 bits rounds to nearest even.
template <class T, int N>
struct Vec {
  typedef T raw __attribute__((ext_vector_type(N)));
};

template <class T, int N>
__device__ __forceinline__ void load(const T* p, float (&x)[N]) {
  constexpr int kPer = 16 / sizeof(T) < N ? 16 / sizeof(T) : N;     // elements of one access
  using V = typename Vec<T, kPer>::raw;
#pragma unroll
  for (int j = 0; j < N / kPer; ++j) {
    const V v = reinterpret_cast<const V*>(p)[j];
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[j * kPer + i] = static_cast<float>(v[i]);
  }
}

template <class T, int N>
__device__ __forceinline__ void store(T* p, const float (&x)[N]) {
  constexpr int kPer = 16 / sizeof(T) < N ? 16 / sizeof(T) : N;
  using V = typename Vec<T, kPer>::raw;
#pragma unroll
  for (int j = 0; j < N / kPer; ++j) {
    V v;
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = static_cast<T>(x[j * kPer + i]);
    reinterpret_cast<V*>(p)[j] = v;
  }
}

// Streams: accesses relative to an address that is the same for the whole wave, through
// buffer instructions, whose cache policy is explicit: kNt is not kept in the caches.
constexpr int kNt = 2;

struct Stream {
  __amdgpu_buffer_rsrc_t r;
  // 0x00020000: raw (unformatted) 32-bit buffer accesses on gfx9
  __device__ __forceinline__ Stream(const void* base, uint32_t bytes)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, static_cast<int>(bytes), 0x00020000)) {}

  template <int P, int BYTES>
  __device__ __forceinline__ auto get(uint32_t at) const {
    if constexpr (BYTES == 16)
      return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, P);
    else if constexpr (BYTES == 8)
      return __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, P);
    else
      return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, P);
  }
  template <int P, class V>
  __device__ __forceinline__ void put(uint32_t at, V v) const {
    if constexpr (sizeof(V) == 16)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, at, 0, P);
    else if constexpr (sizeof(V) == 8)
      __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), r, at, 0, P);
    else
      __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), r, at, 0, P);
  }

  // N values of type T from byte `at` on, as fp32 and back
  template <class T, int P, int N>
  __device__ __forceinline__ void load(uint32_t at, float (&x)[N]) const {
    constexpr int kPer = 16 / sizeof(T) < N ? 16 / sizeof(T) : N;
    using V = typename Vec<T, kPer>::raw;
#pragma unroll
    for (int j = 0; j < N / kPer; ++j) {
      const V v = __builtin_bit_cast(V, get<P, kPer * sizeof(T)>(at + j * kPer * sizeof(T)));
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[j * kPer + i] = static_cast<float>(v[i]);
    }
  }
  template <class T, int P, int N>
  __device__ __forceinline__ void store(uint32_t at, const float (&x)[N]) const {
    constexpr int kPer = 16 / sizeof(T) < N ? 16 / sizeof(T) : N;
    using V = typename Vec<T, kPer>::raw;
#pragma unroll
    for (int j = 0; j < N / kPer; ++j) {
      V v;
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = static_cast<T>(x[j * kPer + i]);
      put<P>(at + j * kPer * sizeof(T), v);
    }
  }
};

// ---------------------------------------------------------------- cross-lane steps
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// The value of the partner lane in step LEVEL of a butterfly over 2^(LEVEL+1)
// lanes: neighbours, pairs, quads (mirrored inside 8) and eights (mirrored
// inside 16); mirrors do where all lanes of a quad, or of an eight, agree.
template <int LEVEL>
__device__ __forceinline__ float partner(float x) {
  static_assert(LEVEL >= 0 && LEVEL < 4, "inside a row of 16 lanes");
  constexpr int kCtrl[4] = {0xb1 /* quad_perm 1,0,3,2 */, 0x4e /* 2,3,0,1 */, 0x141 /* row_half_mirror */, 0x140 /* row_mirror */};
  return dpp<kCtrl[LEVEL]>(x);
}

// Both halves' values of a wave's 32-lane (or, in each of those, 16-lane) halves.
struct Two {
  float a, b;
};
__device__ __forceinline__ Two halves32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a = r[0], b = r[1];      // a bit cast of a vector's element takes its first
  return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ Two halves16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t a = r[0], b = r[1];      // a bit cast of a vector's element takes its first
  return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

template <int LEVELS, class F>
__device__ __forceinline__ float across(float x, F f) {
  if constexpr (LEVELS > 0) x = f(x, partner<0>(x));
  if constexpr (LEVELS > 1) x = f(x, partner<1>(x));
  if constexpr (LEVELS > 2) x = f(x, partner<2>(x));
  if constexpr (LEVELS > 3) x = f(x, partner<3>(x));
  if constexpr (LEVELS > 4) {
    const Two t = halves16(x);
    x = f(t.a, t.b);
  }
  if constexpr (LEVELS > 5) {
    const Two t = halves32(x);
    x = f(t.a, t.b);
  }
  return x;
}

// The sum over a wave, the same in every lane.
__device__ __forceinline__ int wave_sum(int x) {
  const float sum = across<6>(__builtin_bit_cast(float, x), [](float p, float q) {
    return __builtin_bit_cast(float, __builtin_bit_cast(int, p) + __builtin_bit_cast(int, q));
  });
  return __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, sum));
}

// x / n for 0 <= x < 2^31: the high half of a product with 2^32 / n rounded up is at
// most one too many.
struct Divisor {
  uint32_t n, inverse;
  __device__ __forceinline__ int divide(int x) const {
    if (n == 1) return x;
    const uint32_t q = __umulhi(static_cast<uint32_t>(x), inverse);
    return static_cast<int>(q * n > static_cast<uint32_t>(x) ? q - 1 : q);
  }
};

inline Divisor divisor(int n) { return {static_cast<uint32_t>(n), static_cast<uint32_t>(((uint64_t{1} << 32) + n - 1) / n)}; }

// ---------------------------------------------------------------- host side
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Compute units of the current device, read once per device.
inline int device_cus() {
  static std::atomic<int> cache[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) dev = -1;
  if (dev >= 0 && dev < 64) {
    const int c = cache[dev].load(std::memory_order_relaxed);
    if (c > 0) return c;
  }
  int c = 0;
  if (dev < 0 || hipDeviceGetAttribute(&c, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || c <= 0) c = 256;
  if (dev >= 0 && dev < 64) cache[dev].store(c, std::memory_order_relaxed);
  return c;
}

// The stream must belong to the current device.
inline int check_stream_device(hipStream_t stream) {
  int current = 0;
  hipDevice_t owner = 0;
  if (hipGetDevice(&current) != hipSuccess || hipStreamGetDevice(stream, &owner) != hipSuccess) return FEWBIT_E_HIP;
  return owner == current ? FEWBIT_OK : FEWBIT_E_INVALID;
}

// A launch has fewer than 2^32 threads.
constexpr int64_t kThreadsLaunch = int64_t{1} << 32;
inline bool fits_launch(int64_t groups, int64_t threads) { return groups < kThreadsLaunch / threads; }

// A launch by the runtime's own call, which returns its status.
template <class T>
struct Same {
  using type = T;
};
template <class... P>
hipError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t stream, typename Same<P>::type... args) {
  void* pointers[] = {const_cast<void*>(static_cast<const void*>(&args))...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), pointers, 0, stream);
}

// Status of a launch; with FEWBIT_DEBUG set in the environment the HIP error
// behind FEWBIT_E_HIP is printed to stderr.
inline int launch_status(const char* where, hipError_t e) {
  if (e == hipSuccess) return FEWBIT_OK;
  (void)hipGetLastError();          // not left for the caller's next query
  if (std::getenv("FEWBIT_DEBUG"))
    std::fprintf(stderr, "fewbit: %s launch failed: %s (%s)\n", where, hipGetErrorName(e), hipGetErrorString(e));
  return FEWBIT_E_HIP;
}

}  // namespace block
