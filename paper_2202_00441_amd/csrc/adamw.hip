// adamw.hip -- one AdamW step over many tensors, moments in 32 or in 8 bits.
//
// The formulas and the 8-bit format are in fewbit_block.h.  The step is bound by
// HBM: per element it reads and writes a parameter and two moments and reads a
// gradient (bf16 with 8-bit moments: 10 bytes; fp32 with 32-bit ones: 28).  10^8 elements:
//   bf16, 8-bit moments                    170 us   5.9 TB/s
//   bf16, 8-bit moments, master copy       261      6.1
//   fp32, 8-bit moments                    255      6.3
//   bf16, 32-bit moments                   359      6.1
//   fp32, 32-bit moments                   462      6.1
//
// A workgroup takes 16 blocks of 256 elements of one tensor, found in the list that
// travels as kernel arguments, and ends: the dispatcher balances the compute units.
// With 8-bit moments 32 lanes hold a block, eight elements each (8 bytes of codes, 16 of
// a 16-bit parameter), and find the block's largest magnitudes by cross-lane steps;
// with 32-bit ones 64 lanes hold it, four elements each (16 bytes).
//
// Roundings.  Moments, root and update are fp32; sums of products are not fused,
// so that the two moments are the same on every implementation of the formulas,
// and so are the block scales, which are powers of two and change by a factor of
// two where a largest magnitude crosses a bound.  The root and the quotient of
// the update are the hardware's approximations (1 ulp each): what they feed is
// added to a weight some thousand times as large.
#include <algorithm>

#include "block.h"

namespace {

using namespace block;

constexpr int kBlock = FEWBIT_ADAMW_BLOCK;
constexpr int kThreads = 512;
constexpr int kMaxTensors = 256;    // of one launch: their list is 9 KB of arguments
// Blocks of a workgroup (eight in 256 threads: 3 to 5% slower with a master copy or 32-bit
// moments) and the streams' cache policy (10^8 bf16 elements with a master copy and 8-bit
// moments: 261 us, with loads alone past the caches 293, with neither 294).
constexpr int kRun = 16;
constexpr int kLoad = kNt, kStore = kNt;

struct Tensor {
  void* p;
  const void* g;
  int64_t n;
  int64_t block0;       // its first block in the flat buffers
};

struct Args {
  Tensor t[kMaxTensors];
  uint32_t first[kMaxTensors];      // its first workgroup
  int count;
  void *m, *v;
  float *ms, *vs, *master;
  float b1, a1, b2, a2;             // betas and 1 - beta
  float keep, step, root, eps;      // 1 - lr decay; lr / (1 - beta1^t); 1 / sqrt(1 - beta2^t)
  uint32_t key;
};

// The update of N elements; codes and scales apart.
template <int N>
__device__ __forceinline__ void moments(const Args& a, const float (&g)[N], float (&m)[N], float (&v)[N]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    m[i] = m[i] * a.b1 + g[i] * a.a1;
    v[i] = v[i] * a.b2 + (g[i] * g[i]) * a.a2;
  }
}
// SMALL: what the hardware's root takes as 0, moments below the normal range, is brought into
// its range first.
template <bool SMALL, int N>
__device__ __forceinline__ void update(const Args& a, float (&w)[N], const float (&g)[N], float (&m)[N], float (&v)[N]) {
  moments(a, g, m, v);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool below = SMALL && v[i] < 0x1p-126f;
    const float root = __builtin_amdgcn_sqrtf(below ? v[i] * 0x1p64f : v[i]) * (below ? 0x1p-32f : 1.0f);
    const float d = root * a.root + a.eps;
    w[i] = w[i] * a.keep - a.step * (m[i] * __builtin_amdgcn_rcpf(d));
  }
}

// A block's largest magnitude over the 32 lanes that hold it.  Infinities and NaN are left
// out: they become NaN codes whatever the scale, and infinities here, for adding the dither
// to a NaN's mantissa may carry into its sign.
template <int N>
__device__ __forceinline__ float largest(float (&x)[N]) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) most = __builtin_elementwise_maximum(most, fabsf(x[i]));      // a NaN stays one
  if (__builtin_expect(__any(!(most < INFINITY)), 0)) {
    most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (fabsf(x[i]) < INFINITY)
        most = fmaxf(most, fabsf(x[i]));
      else
        x[i] = INFINITY;
    }
  }
  return across<5>(most, [](float p, float q) { return fmaxf(p, q); });
}

// Exponent field of the block's scale: the least power of two 2^e with
// most <= 448 * 2^e = 1.75 * 2^(e + 8), at least 2^-125.
__device__ __forceinline__ uint32_t scale_field(float most) {
  const uint32_t b = __builtin_bit_cast(uint32_t, fmaxf(most, 0x1p-117f));
  return (b >> 23) - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);
}
__device__ __forceinline__ float power(uint32_t field) { return __builtin_bit_cast(float, field << 23); }

// y >= 0 (at most 448, or infinite) rounded to one of the two 8-bit numbers around it,
// up with the probability of its distance from the lower: u / 2^16 of that or more is
// taken up.  The format keeps three bits of 23 behind the leading one; adding u to the
// 16 bits below them carries into them as it should.  Below 2^-6 its numbers are 2^-9
// apart, as those of the binade from 2^-6 on are: there y takes the detour through that.
__device__ __forceinline__ float dithered(float y, uint32_t u) {
  const float detour = y < 0x1p-6f ? 0x1p-6f : 0.0f;
  const uint32_t bits = __builtin_bit_cast(uint32_t, y + detour) + (u << 4);
  return __builtin_bit_cast(float, bits & 0xfff00000u) - detour;
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

template <int N>
__device__ __forceinline__ void unpack(const uint32_t (&c)[N / 4], float scale, float (&x)[N]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[j], true);
    x[4 * j] = lo[0] * scale;
    x[4 * j + 1] = lo[1] * scale;
    x[4 * j + 2] = hi[0] * scale;
    x[4 * j + 3] = hi[1] * scale;
  }
}

// N elements from byte `at` on, of which `left` are there; the others read as 0 and are
// not written.  `whole`: all of them are, and the address is aligned.
template <class T, int N>
__device__ __forceinline__ void load_some(const Stream& s, const T* base, uint32_t at, int64_t left, bool whole, float (&x)[N]) {
  if (whole) return s.load<T, kLoad>(at, x);
  const T* p = reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + at);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = i < left ? static_cast<float>(p[i]) : 0.0f;
}
template <class T, int N>
__device__ __forceinline__ void store_some(const Stream& s, T* base, uint32_t at, int64_t left, bool whole, const float (&x)[N]) {
  if (whole) return s.store<T, kStore>(at, x);
  T* p = reinterpret_cast<T*>(reinterpret_cast<char*>(base) + at);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < left) p[i] = static_cast<T>(x[i]);
}

// The moments of N elements, as codes of a block that 32 lanes hold; the second four of
// a lane's elements lie `apart` elements behind its first.
template <int N>
__device__ __forceinline__ void encode(const Args& a, int64_t flat, int apart, float (&m)[N], float (&v)[N], uint32_t (&cm)[N / 4],
                                       uint32_t (&cv)[N / 4], float& ms, float& vs) {
  const uint32_t fm = scale_field(largest(m)), fv = scale_field(largest(v));
  const float im = power(254 - fm), iv = power(254 - fv);
  float rm[N], rv[N];
  const uint32_t first = static_cast<uint32_t>(flat) * 0x9E3779B1u + a.key;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t x = first + static_cast<uint32_t>(i / 4 * apart + i % 4) * 0x9E3779B1u;
    uint32_t h = (x ^ x >> 15) * 0xBB67AE85u;
    h ^= h >> 13;
    rm[i] = copysignf(dithered(fabsf(m[i]) * im, h >> 16), m[i]);
    rv[i] = dithered(v[i] * iv, h & 0xffff);
    if (v[i] > 0.0f) rv[i] = fmaxf(rv[i], 0x1p-9f);
  }
#pragma unroll
  for (int j = 0; j < N / 4; ++j) {
    cm[j] = pack4(rm[4 * j], rm[4 * j + 1], rm[4 * j + 2], rm[4 * j + 3]);
    cv[j] = pack4(rv[4 * j], rv[4 * j + 1], rv[4 * j + 2], rv[4 * j + 3]);
  }
  ms = power(fm);
  vs = power(fv);
}

template <int PT, int GT, int BITS, bool MASTER, bool SMALL>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Args a) {
  using P = typename Store<PT>::type;
  using G = typename Store<GT>::type;
  constexpr int N = BITS == 8 ? 8 : 4;              // elements of a lane in a row
  constexpr int kLanes = kBlock / N;                // lanes of a block

  // the tensor: the last whose first workgroup is not past this one
  const int l = threadIdx.x % kWave;
  int before = 0;
#pragma unroll
  for (int i = 0; i < kMaxTensors; i += kWave) {
    const uint32_t first = a.first[i + l];
    before += __builtin_popcountll(__ballot(i + l < a.count && first <= blockIdx.x));
  }
  const Tensor t = a.t[__builtin_amdgcn_readfirstlane(before - 1)];
  const int64_t block = static_cast<int64_t>(blockIdx.x - a.first[__builtin_amdgcn_readfirstlane(before - 1)]) * kRun;   // the first, of the tensor's
  const bool aligned = ((reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(t.g)) & 15) == 0;
  P* p = static_cast<P*>(t.p) + block * kBlock;
  const G* g = static_cast<const G*>(t.g) + block * kBlock;
  const int64_t flat = (t.block0 + block) * kBlock, left = t.n - block * kBlock;
  constexpr uint32_t kAll = kRun * kBlock;
  const Stream sp(p, kAll * sizeof(P)), sg(g, kAll * sizeof(G)), sw(a.master + flat, kAll * 4);
  if constexpr (BITS == 32) {
    // every lane has four elements in each of its wave's two blocks
    const Stream sm(static_cast<float*>(a.m) + flat, kAll * 4), sv(static_cast<float*>(a.v) + flat, kAll * 4);
    constexpr int kRows = kRun * kLanes / kThreads;
    float w[kRows][N], gr[kRows][N], m[kRows][N], v[kRows][N];
    uint32_t at[kRows];
    bool whole[kRows], some[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      at[r] = ((threadIdx.x / kWave * kRows + r) * kWave + l) * N;
      whole[r] = aligned && left - at[r] >= N;
      some[r] = at[r] / kBlock * kBlock < left;       // of all lanes of the block alike
      if (!some[r]) continue;
      load_some(sg, g, at[r] * sizeof(G), left - at[r], whole[r], gr[r]);
      sm.load<float, kLoad>(at[r] * 4, m[r]);
      sv.load<float, kLoad>(at[r] * 4, v[r]);
      if constexpr (MASTER)
        sw.load<float, kLoad>(at[r] * 4, w[r]);
      else
        load_some<P>(sp, p, at[r] * sizeof(P), left - at[r], whole[r], w[r]);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (!some[r]) continue;
      update<SMALL>(a, w[r], gr[r], m[r], v[r]);
      sm.store<float, kStore>(at[r] * 4, m[r]);
      sv.store<float, kStore>(at[r] * 4, v[r]);
      if constexpr (MASTER) sw.store<float, kStore>(at[r] * 4, w[r]);
      store_some(sp, p, at[r] * sizeof(P), left - at[r], whole[r], w[r]);
    }
  } else {
    // A lane's eight elements lie side by side where that is 16 bytes of everything;
    // with a stream of fp32 in two rows of four, each of which 32 lanes fill.
    constexpr int kApart = PT != FEWBIT_F32 && GT != FEWBIT_F32 && !MASTER ? 4 : kBlock / 2;
    constexpr int kRow = kApart == 4 ? N : 4, kRows = N / kRow;
    const uint32_t at = threadIdx.x / kLanes * kBlock + threadIdx.x % kLanes * kRow;
    if (at / kBlock * kBlock >= left) return;         // all lanes of the block alike
    const Stream sm(static_cast<uint8_t*>(a.m) + flat, kAll), sv(static_cast<uint8_t*>(a.v) + flat, kAll);
    const int64_t b = t.block0 + block + at / kBlock;
    float w[kRows][kRow], gr[N], m[N], v[N], wf[N];
    uint32_t qm[N / 4], qv[N / 4];
    bool whole[kRows];
    if constexpr (kRows == 1) {
      const u32x2 x = sm.get<kLoad, 8>(at), y = sv.get<kLoad, 8>(at);
      qm[0] = x[0], qm[1] = x[1], qv[0] = y[0], qv[1] = y[1];
    } else {
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        qm[r] = sm.get<kLoad, 4>(at + r * kApart);
        qv[r] = sv.get<kLoad, 4>(at + r * kApart);
      }
    }
    const float oldm = a.ms[b], oldv = a.vs[b];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const uint32_t here = at + r * kApart;
      float x[kRow];
      whole[r] = aligned && left - here >= kRow;
      load_some(sg, g, here * sizeof(G), left - here, whole[r], x);
      if constexpr (MASTER)
        sw.load<float, kLoad>(here * 4, w[r]);
      else
        load_some<P>(sp, p, here * sizeof(P), left - here, whole[r], w[r]);
#pragma unroll
      for (int i = 0; i < kRow; ++i) {
        gr[r * kRow + i] = x[i];
        wf[r * kRow + i] = w[r][i];
      }
    }
    unpack<N>(qm, oldm, m);
    unpack<N>(qv, oldv, v);
    update<SMALL>(a, wf, gr, m, v);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const uint32_t here = at + r * kApart;
#pragma unroll
      for (int i = 0; i < kRow; ++i) w[r][i] = wf[r * kRow + i];
      if constexpr (MASTER) sw.store<float, kStore>(here * 4, w[r]);
      store_some(sp, p, here * sizeof(P), left - here, whole[r], w[r]);
    }
    float ms, vs;
    encode(a, flat + at, kApart, m, v, qm, qv, ms, vs);
    if constexpr (kRows == 1) {
      sm.put<kStore>(at, u32x2{qm[0], qm[1]});
      sv.put<kStore>(at, u32x2{qv[0], qv[1]});
    } else {
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        sm.put<kStore>(at + r * kApart, qm[r]);
        sv.put<kStore>(at + r * kApart, qv[r]);
      }
    }
    if (at % kBlock == 0) {
      a.ms[b] = ms;
      a.vs[b] = vs;
    }
  }
}

template <int PT, int GT, int BITS, bool MASTER>
hipError_t start_small(const Args& a, unsigned groups, hipStream_t s) {
  // Roots that the hardware takes as 0 are below 2^-63: where the denominator's eps does not
  // hide them they are formed with care.  (Always: 700 us where 684, 8 layers of width 2048 in
  // bf16 with 8-bit moments.)
  return a.root * 0x1p-63f > a.eps * 0x1p-24f ? launch(adamw_kernel<PT, GT, BITS, MASTER, true>, dim3(groups), kThreads, s, a)
                                              : launch(adamw_kernel<PT, GT, BITS, MASTER, false>, dim3(groups), kThreads, s, a);
}

template <int PT, int GT, int BITS>
hipError_t start(const Args& a, unsigned groups, hipStream_t s) {
  if constexpr (PT != FEWBIT_F32)
    if (a.master) return start_small<PT, GT, BITS, true>(a, groups, s);
  return start_small<PT, GT, BITS, false>(a, groups, s);
}

template <int PT, int GT>
hipError_t start_bits(const Args& a, int bits, unsigned groups, hipStream_t s) {
  return bits == 8 ? start<PT, GT, 8>(a, groups, s) : start<PT, GT, 32>(a, groups, s);
}

template <int PT>
hipError_t start_grad(const Args& a, int gt, int bits, unsigned groups, hipStream_t s) {
  return gt == PT ? start_bits<PT, PT>(a, bits, groups, s) : start_bits<PT, FEWBIT_F32>(a, bits, groups, s);
}

int64_t blocks_of(int64_t n) { return n / kBlock + (n % kBlock != 0); }

}  // namespace

extern "C" int fewbit_adamw_step(const fewbit_adamw* h, const fewbit_adamw_tensor* tensors, int32_t count, void* m,
                                 void* v, float* m_scale, float* v_scale, float* master, void* stream) {
  if (!h) return FEWBIT_E_NULL;
  const int pt = h->param_dtype, gt = h->grad_dtype;
  if (pt < FEWBIT_F32 || pt > FEWBIT_BF16 || (gt != pt && gt != FEWBIT_F32)) return FEWBIT_E_DTYPE;
  if (h->state_bits != 8 && h->state_bits != 32) return FEWBIT_E_BITS;
  if (count < 0 || h->reserved != 0 || h->step < 1) return FEWBIT_E_INVALID;
  if (!(h->lr >= 0.0 && std::isfinite(h->lr)) || !(h->beta1 >= 0.0 && h->beta1 < 1.0) ||
      !(h->beta2 >= 0.0 && h->beta2 < 1.0) || !(h->eps >= 0.0 && std::isfinite(h->eps)) ||
      !(h->weight_decay >= 0.0 && std::isfinite(h->weight_decay)))
    return FEWBIT_E_INVALID;
  if (master && pt == FEWBIT_F32) return FEWBIT_E_INVALID;          // the parameters are one
  if (count == 0) return FEWBIT_OK;
  if (!tensors) return FEWBIT_E_NULL;
  int64_t total = 0;
  for (int i = 0; i < count; ++i) {
    if (tensors[i].n < 0 || tensors[i].n >= int64_t{1} << 40) return FEWBIT_E_INVALID;
    if (tensors[i].n > 0 && tensors[i].grad && !tensors[i].param) return FEWBIT_E_NULL;
    total += blocks_of(tensors[i].n);
  }
  if (total == 0) return FEWBIT_OK;
  if (!m || !v || (h->state_bits == 8 && (!m_scale || !v_scale))) return FEWBIT_E_NULL;
  if (misaligned(m) || misaligned(v) || misaligned(m_scale) || misaligned(v_scale) || misaligned(master))
    return FEWBIT_E_ALIGN;
  const int rc = check_stream_device(static_cast<hipStream_t>(stream));
  if (rc != FEWBIT_OK) return rc;

  Args a;
  a.m = m;
  a.v = v;
  a.ms = m_scale;
  a.vs = v_scale;
  a.master = master;
  a.b1 = static_cast<float>(h->beta1);
  a.a1 = static_cast<float>(1.0 - h->beta1);
  a.b2 = static_cast<float>(h->beta2);
  a.a2 = static_cast<float>(1.0 - h->beta2);
  const double t = static_cast<double>(h->step);
  a.keep = static_cast<float>(1.0 - h->lr * h->weight_decay);
  a.step = static_cast<float>(h->lr / (1.0 - std::pow(h->beta1, t)));
  a.root = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t)));
  a.eps = static_cast<float>(h->eps);
  a.key = static_cast<uint32_t>(h->seed) * 0x6A09E667u + 0x3C6EF372u;

  const hipStream_t s = static_cast<hipStream_t>(stream);
  constexpr int64_t kGroupsMost = kThreadsLaunch / kThreads - 1;
  int64_t groups = 0;
  a.count = 0;
  const auto start = [&]() {
    if (a.count == 0) return static_cast<int>(FEWBIT_OK);
    const unsigned n = static_cast<unsigned>(groups);
    const hipError_t e = pt == FEWBIT_F32   ? start_grad<FEWBIT_F32>(a, gt, h->state_bits, n, s)
                         : pt == FEWBIT_F16 ? start_grad<FEWBIT_F16>(a, gt, h->state_bits, n, s)
                                            : start_grad<FEWBIT_BF16>(a, gt, h->state_bits, n, s);
    a.count = 0;
    groups = 0;
    return launch_status("fewbit_adamw_step", e);
  };
  // A tensor that the rest of a launch does not hold goes on in the next, after whole workgroups.
  const int64_t p_size = pt == FEWBIT_F32 ? 4 : 2, g_size = gt == FEWBIT_F32 ? 4 : 2;
  int64_t block0 = 0;
  for (int i = 0; i < count; ++i) {
    const int64_t blocks = blocks_of(tensors[i].n);
    for (int64_t b = 0; b < blocks && tensors[i].grad;) {
      if (a.count == kMaxTensors || groups == kGroupsMost) {
        const int status = start();
        if (status != FEWBIT_OK) return status;
      }
      const int64_t take = std::min(blocks - b, (kGroupsMost - groups) * kRun), at = b * kBlock;
      a.t[a.count] = {static_cast<char*>(tensors[i].param) + at * p_size, static_cast<const char*>(tensors[i].grad) + at * g_size,
                      tensors[i].n - at, block0 + b};
      a.first[a.count++] = static_cast<uint32_t>(groups);
      groups += (take + kRun - 1) / kRun;
      b += take;
    }
    block0 += blocks;
  }
  return start();
}
