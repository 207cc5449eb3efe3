// adamw.hip -- one AdamW step over many tensors, moments in 32 or in 8 bits.
//
// The formulas and the 8-bit format are in fewbit_block.h.  The step is bound by
// HBM: per element it reads and writes a parameter and two moments and reads a
// gradient (bf16 with 8-bit moments: 10 bytes; fp32 with 32-bit ones: 28).
//
// A workgroup takes a run of 256-element blocks of one tensor, found in the list
// that travels as kernel arguments; its waves take blocks in turn.  With 8-bit
// moments 32 lanes hold a block, eight elements each (8 bytes of codes, 16 of a
// 16-bit parameter), and find the block's largest magnitudes by cross-lane
// steps; with 32-bit ones 64 lanes hold it, four elements each (16 bytes).
//
// Roundings.  Moments, root and update are fp32; sums of products are not fused,
// so that the two moments are the same on every implementation of the formulas,
// and so are the block scales, which are powers of two and change by a factor of
// two where a largest magnitude crosses a bound.  The root and the quotient of
// the update are the hardware's approximations (1 ulp each): what they feed is
// added to a weight some thousand times as large.
#include "block.h"

namespace {

using namespace block;

constexpr int kBlock = FEWBIT_ADAMW_BLOCK;
constexpr int kThreads = 256;
constexpr int kMaxTensors = 96;     // of one launch: their list is 3 KB of arguments

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
  int run;              // blocks of a workgroup
  void *m, *v;
  float *ms, *vs, *master;
  float b1, a1, b2, a2;             // betas and 1 - beta
  float keep, step, root, eps;      // 1 - lr decay; lr / (1 - beta1^t); 1 / sqrt(1 - beta2^t)
  uint32_t key;
};

// The update of N elements; codes and scales apart.
template <int N>
__device__ __forceinline__ void update(const Args& a, float (&w)[N], const float (&g)[N], float (&m)[N], float (&v)[N]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    m[i] = m[i] * a.b1 + g[i] * a.a1;
    v[i] = v[i] * a.b2 + (g[i] * g[i]) * a.a2;
    const float d = __builtin_amdgcn_sqrtf(v[i]) * a.root + a.eps;
    w[i] = w[i] * a.keep - a.step * (m[i] * __builtin_amdgcn_rcpf(d));
  }
}

// A block's largest magnitude over the 32 lanes that hold it, infinities and NaN
// left out (they become NaN codes whatever the scale).
template <int N>
__device__ __forceinline__ float largest(const float (&x)[N]) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(x[i]));
  if (__builtin_expect(__any(!(most < INFINITY)), 0)) {
    most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.0f);
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

// y >= 0 (at most 448, or not finite) rounded to one of the two 8-bit numbers
// around it, up with probability of its distance from the lower: u in [0, 1).
// y is counted in steps of its binade (in steps of 2^-9 below 2^-6).
__device__ __forceinline__ float dithered(float y, float u) {
  const uint32_t e = max(__builtin_bit_cast(uint32_t, y) >> 23, 121u);
  return floorf(y * power(257 - e) + u) * power(e - 3);
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

// N elements from p on, of which `left` are there; the others read as 0 and are
// not written.  `whole`: all of them are, and p is aligned.
template <class T, int N>
__device__ __forceinline__ void load_some(const T* p, int64_t left, bool whole, float (&x)[N]) {
  if (whole) return load(p, x);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = i < left ? static_cast<float>(p[i]) : 0.0f;
}
template <class T, int N>
__device__ __forceinline__ void store_some(T* p, int64_t left, bool whole, const float (&x)[N]) {
  if (whole) return store(p, x);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < left) p[i] = static_cast<T>(x[i]);
}

template <int PT, int GT, int BITS, bool MASTER>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Args a) {
  using P = typename Store<PT>::type;
  using G = typename Store<GT>::type;
  constexpr int N = BITS == 8 ? 8 : 4;              // elements of a lane
  constexpr int kLanes = kBlock / N;                // lanes of a block
  constexpr int kStep = kThreads / kLanes;          // blocks of a workgroup's pass

  // the tensor: the last whose first workgroup is not past this one
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    (a.first[mid] <= blockIdx.x ? lo : hi) = mid;
  }
  const Tensor t = a.t[lo];
  const int64_t start = static_cast<int64_t>(blockIdx.x - a.first[lo]) * a.run;     // in the tensor's blocks
  const bool aligned = ((reinterpret_cast<uintptr_t>(t.p) | reinterpret_cast<uintptr_t>(t.g)) & 15) == 0;
  const int lane = threadIdx.x % kLanes;
  for (int64_t b = start + threadIdx.x / kLanes, end = start + a.run; b < end; b += kStep) {
    const int64_t at = b * kBlock + lane * N, left = t.n - at;
    if (b * kBlock >= t.n) break;                   // of all lanes of the block alike
    const bool whole = aligned && left >= N;
    const int64_t flat = (t.block0 + b) * kBlock + lane * N;
    float w[N], g[N], m[N], v[N];
    load_some(static_cast<const G*>(t.g) + at, left, whole, g);
    if constexpr (MASTER)
      load(a.master + flat, w);
    else
      load_some(static_cast<const P*>(t.p) + at, left, whole, w);
    if constexpr (BITS == 32) {
      load(static_cast<const float*>(a.m) + flat, m);
      load(static_cast<const float*>(a.v) + flat, v);
      update(a, w, g, m, v);
      store(static_cast<float*>(a.m) + flat, m);
      store(static_cast<float*>(a.v) + flat, v);
    } else {
      u32x2* cm = reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.m) + flat);
      u32x2* cv = reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.v) + flat);
      const u32x2 qm = *cm, qv = *cv;
      unpack<N>({qm[0], qm[1]}, a.ms[t.block0 + b], m);
      unpack<N>({qv[0], qv[1]}, a.vs[t.block0 + b], v);
      update(a, w, g, m, v);
      const uint32_t fm = scale_field(largest(m)), fv = scale_field(largest(v));
      const float im = power(254 - fm), iv = power(254 - fv);
      float rm[N], rv[N];
      uint32_t x = static_cast<uint32_t>(flat) * 0x9E3779B1u + a.key;
#pragma unroll
      for (int i = 0; i < N; ++i, x += 0x9E3779B1u) {
        uint32_t h = (x ^ x >> 15) * 0xBB67AE85u;
        h ^= h >> 13;
        rm[i] = copysignf(dithered(fabsf(m[i]) * im, static_cast<float>(h >> 16) * 0x1p-16f), m[i]);
        rv[i] = dithered(v[i] * iv, static_cast<float>(h & 0xffff) * 0x1p-16f);
        if (v[i] > 0.0f) rv[i] = fmaxf(rv[i], 0x1p-9f);
      }
      *cm = u32x2{pack4(rm[0], rm[1], rm[2], rm[3]), pack4(rm[4], rm[5], rm[6], rm[7])};
      *cv = u32x2{pack4(rv[0], rv[1], rv[2], rv[3]), pack4(rv[4], rv[5], rv[6], rv[7])};
      if (lane == 0) {
        a.ms[t.block0 + b] = power(fm);
        a.vs[t.block0 + b] = power(fv);
      }
    }
    if constexpr (MASTER) store(a.master + flat, w);
    store_some(static_cast<P*>(t.p) + at, left, whole, w);
  }
}

template <int PT, int GT, int BITS>
hipError_t start(const Args& a, unsigned groups, hipStream_t s) {
  if constexpr (PT != FEWBIT_F32)
    if (a.master) return launch(adamw_kernel<PT, GT, BITS, true>, dim3(groups), kThreads, s, a);
  return launch(adamw_kernel<PT, GT, BITS, false>, dim3(groups), kThreads, s, a);
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
  // Blocks of a workgroup: enough for eight passes where that still gives the
  // chip eight workgroups per CU, one pass at least.
  const int64_t wanted = total / (8 * static_cast<int64_t>(device_cus()));
  a.run = wanted >= 64 ? 64 : wanted >= 32 ? 32 : wanted >= 16 ? 16 : 8;

  int64_t block0 = 0;
  for (int i = 0; i < count;) {
    uint64_t groups = 0;
    a.count = 0;
    for (; i < count && a.count < kMaxTensors; ++i) {
      const int64_t blocks = blocks_of(tensors[i].n);
      if (blocks == 0 || !tensors[i].grad) {
        block0 += blocks;
        continue;
      }
      const uint64_t more = (blocks + a.run - 1) / a.run;
      if (groups + more >= uint64_t{1} << 24) {                      // fewer than 2^32 threads
        if (a.count == 0) return FEWBIT_E_INVALID;                   // more than any device's memory holds
        break;
      }
      a.t[a.count] = {tensors[i].param, tensors[i].grad, tensors[i].n, block0};
      a.first[a.count++] = static_cast<uint32_t>(groups);
      groups += more;
      block0 += blocks;
    }
    if (a.count == 0) continue;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned n = static_cast<unsigned>(groups);
    const hipError_t e = pt == FEWBIT_F32   ? start_grad<FEWBIT_F32>(a, gt, h->state_bits, n, s)
                         : pt == FEWBIT_F16 ? start_grad<FEWBIT_F16>(a, gt, h->state_bits, n, s)
                                            : start_grad<FEWBIT_BF16>(a, gt, h->state_bits, n, s);
    const int status = launch_status("fewbit_adamw_step", e);
    if (status != FEWBIT_OK) return status;
  }
  return FEWBIT_OK;
}
