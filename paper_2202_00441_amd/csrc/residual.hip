// residual.hip -- dropout from a counter, the addition of a branch to the residual stream
// with the RMS norm of the sum (in the storage type or in 8 bits), rows in 8 bits, and the
// gradients.
//
// Formulas in fewbit_residual.h.  All are bound by HBM: each element is read once and each
// result written once.
//
// A row of the norm is held in registers by 1, 4 or 16 waves, up to 4 chunks of eight
// elements to a lane, so that its sum is known before any of it is read again.  Rows are
// reached through buffer accesses whose range is the row: chunks past its end read zeros
// and write nothing.
#include <algorithm>
#include <type_traits>

#include "drop.h"

namespace {

using namespace block;

// ---------------------------------------------------------------- dropout
constexpr int kDropThreads = 256;
constexpr int kDropBlocks = 4;      // blocks of eight elements of a lane

// 32768 x 2048 bf16: 42 us, 6.4 TB/s; a copy of the same bytes reaches 6.6.
template <int DT>
__global__ __launch_bounds__(kDropThreads) void drop_kernel(const void* x, void* y, int64_t n, const Drop d) {
  using T = typename Store<DT>::type;
  constexpr int kBytes = 8 * sizeof(T);
  constexpr int kTile = kWave * kDropBlocks;
  const int64_t tile = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) + static_cast<int64_t>(blockIdx.x) * (kDropThreads / kWave);
  const int64_t first = tile * kTile, whole = n / 8;
  const int lane = threadIdx.x % kWave;
  if (first > whole) return;
  const Key key = key_of(d);
  const uint32_t here = static_cast<uint32_t>(min(whole - first, static_cast<int64_t>(kTile)));
  const Stream in(static_cast<const T*>(x) + first * 8, here * kBytes), out(static_cast<T*>(y) + first * 8, here * kBytes);
  float v[kDropBlocks][8];
#pragma unroll
  for (int j = 0; j < kDropBlocks; ++j) Chunk<T>::template load<kNt>(in, j * kWaveElements, lane, v[j]);
#pragma unroll
  for (int j = 0; j < kDropBlocks; ++j) {
    drop<T>(d, key, static_cast<uint64_t>(first + j * kWave), lane, v[j]);
    Chunk<T>::template store<kNt>(out, j * kWaveElements, lane, v[j]);
  }
  // the last n % 8 elements, by the tile that their block falls in
  if (here == kTile || lane >= n % 8) return;
  uint32_t c[4];
  words(static_cast<uint64_t>(whole), key, d.site, c);
  const uint32_t word = lane < 4 ? (lane < 2 ? c[0] : c[1]) : (lane < 6 ? c[2] : c[3]);
  const uint32_t u = lane % 2 ? word >> 16 : word & 0xFFFFu;
  const int64_t at = whole * 8 + lane;
  static_cast<T*>(y)[at] = static_cast<T>(u >= d.border ? scaled<T>(static_cast<float>(static_cast<const T*>(x)[at]), d) : 0.0f);
}

// ---------------------------------------------------------------- rows
// A workgroup of the norm: `WAVES` waves hold a row; below four, each wave has its own.
template <int WAVES>
struct Group {
  static constexpr int kRows = WAVES == 1 ? 4 : 1;
  static constexpr int kThreads = kWave * WAVES * kRows;
};

template <class T>
__device__ __forceinline__ const T* row_of(const void* p, uint32_t row, const Divisor& rows, const int64_t (&s)[2]) {
  const int o = rows.divide(static_cast<int>(row)), i = static_cast<int>(row) - o * static_cast<int>(rows.n);
  return static_cast<const T*>(p) + o * s[0] + i * s[1];
}

// Sums (or largest) over a row of what its lanes hold, the same in every lane.  `parts` is
// not written again before all have passed another barrier.
template <int WAVES, int N, class F>
__device__ __forceinline__ void over_row(float (&x)[N], float (*parts)[N], F f) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = across<6>(x[i], f);
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) parts[wave][i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = parts[0][i];
#pragma unroll
      for (int j = 1; j < WAVES; ++j) x[i] = f(x[i], parts[j][i]);
    }
  }
}

struct Add {
  __device__ float operator()(float a, float b) const { return a + b; }
};
// Of magnitudes, as integers: a NaN is above everything.
struct Largest {
  __device__ float operator()(float a, float b) const {
    return __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)));
  }
};

__device__ __forceinline__ float magnitude(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu); }

struct FwdArgs {
  const void *x, *res, *w;
  void *h, *y;              // y: the norm, or codes
  float* scale;
  int64_t xs[2], rs[2];
  Divisor rows;
  uint32_t total;
  int width;
  float eps;
  Drop drop;
};

enum Out { kNorm, kNorm8, kRows8 };

// Codes of eight elements a (of a row whose largest magnitude is m, inv = 127 / m) as bytes.
// Added to 1.5 * 2^23, t = a inv leaves its nearest whole number, halves to the even, in the
// low bits.  t is off by less than 2^-15 (|t| <= 127 times three roundings): where that leaves
// the code open, 254 |a| is compared with (2 k + 1) m, the border, in 64 bits, exactly for
// 16-bit storage.
template <class A>
__device__ __forceinline__ u32x2 codes_of(const float (&a)[8], const A (&wide)[8], A m, float inv, bool tiny) {
  constexpr float kWhole = 12582912.0f, kOpen = 0.5f - 0x1p-14f;
  uint32_t q[8];
  float off = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float k = fmaf(a[i], inv, kWhole);
    q[i] = __builtin_bit_cast(uint32_t, k);
    off = fmaxf(off, fabsf(fmaf(a[i], inv, kWhole - k)));
  }
  if (off > kOpen || tiny) {
    uint32_t open = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      open |= (tiny || fabsf(fmaf(a[i], inv, kWhole - __builtin_bit_cast(float, q[i]))) > kOpen ? 1u : 0u) << i;
    // one of a lane's eight at a time: seldom more than one in a wave is open
    while (open) {
      const int at = __builtin_ctz(open);
      open &= open - 1;
      float x = a[0];
      A y = wide[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        x = at == i ? a[i] : x;
        y = at == i ? wide[i] : y;
      }
      const double b = fabs(static_cast<double>(y)), top = static_cast<double>(m);
      int k = tiny ? static_cast<int>(127.0 * b / top) : static_cast<int>(fabsf(x) * inv);
      k -= 127.0 * b < k * top;             // t may lie on the other side of a whole number
      const double twice = 254.0 * b, border = (2 * k + 1) * top;
      k += twice > border || (twice == border && (k & 1));
      k = y < 0 ? -k : k;                   // (x may have no sign left)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = at == i ? static_cast<uint32_t>(k) : q[i];
    }
  }
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // the low bytes of four words
    const uint32_t low = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400), high = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x04000c0c);
    r[i] = low | high;
  }
  return r;
}

// 32768 x 2048 bf16: addition, norm and dropout 86 us, 6.3 TB/s, without dropout 85; in 8 bits
// 75 us, 6.3 TB/s; rows of 8192 in 8 bits 126 us, 6.4 TB/s.  One row: 4 us, a launch.
template <int DT, int WAVES, int CHUNKS, Out OUT, bool DROP>
__global__ __launch_bounds__(Group<WAVES>::kThreads) void rnorm_fwd_kernel(const FwdArgs a) {
  using T = typename Store<DT>::type;
  using G = Group<WAVES>;
  // largest products are compared in 64 bits where 32 do not hold them
  constexpr bool kWide = DT == FEWBIT_F32 && OUT == kNorm8;
  using A = typename std::conditional<kWide, double, float>::type;
  using E = Chunk<T>;
  __shared__ float parts[2][WAVES][1];
  __shared__ double wides[WAVES];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t row = blockIdx.x * G::kRows + (WAVES == 1 ? wave : 0);
  if (WAVES == 1 && row >= a.total) return;
  const auto place = [&](int c) __attribute__((always_inline)) { return (c * WAVES + (WAVES == 1 ? 0 : wave)) * kWaveElements; };
  const uint32_t bytes = static_cast<uint32_t>(a.width) * sizeof(T);
  const Stream x(row_of<T>(a.x, row, a.rows, a.xs), bytes);
  float h[CHUNKS][8], w[CHUNKS][8];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) E::template load<kNt>(x, place(c), lane, h[c]);
  if constexpr (OUT != kRows8) {
    const Stream sw(a.w, bytes);
    const int64_t dense = static_cast<int64_t>(row) * a.width;
    const Stream out(static_cast<T*>(a.h) + dense, a.h ? bytes : 0);
    float r[CHUNKS][8];
    const Stream res(a.res ? row_of<T>(a.res, row, a.rows, a.rs) : nullptr, a.res ? bytes : 0);     // none: zeros
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) E::template load<kNt>(res, place(c), lane, r[c]);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) E::template load<0>(sw, place(c), lane, w[c]);
    [[maybe_unused]] const Key key = DROP ? key_of(a.drop) : Key{};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      if constexpr (DROP) drop<T>(a.drop, key, static_cast<uint64_t>((dense + place(c)) / 8), lane, h[c]);
      if (a.res)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] = static_cast<float>(static_cast<T>(h[c][i] + r[c][i]));
      else if (DROP)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] = static_cast<float>(static_cast<T>(h[c][i]));
      E::template store<kNt>(out, place(c), lane, h[c]);
    }
  }
  float size = 1.0f;
  if constexpr (OUT != kRows8) {
    float sum[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[0] += h[c][i] * h[c][i];
    over_row<WAVES>(sum, parts[0], Add());
    size = 1.0f / sqrtf(sum[0] / a.width + a.eps);
  }
  const int64_t dense = static_cast<int64_t>(row) * a.width;
  if constexpr (OUT == kNorm) {
    const Stream y(static_cast<T*>(a.y) + dense, bytes);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * size * w[c][i];
      E::template store<kNt>(y, place(c), lane, h[c]);
    }
  } else {
    float most[1] = {0.0f};
    [[maybe_unused]] double top = 0.0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (kWide) top = fmax(top, fabs(static_cast<double>(h[c][i]) * w[c][i]));
        const float p = OUT == kNorm8 ? h[c][i] * w[c][i] : h[c][i];
        if constexpr (!kWide) h[c][i] = p;
        most[0] = Largest()(most[0], magnitude(p));
      }
    over_row<WAVES>(most, parts[1], Largest());
    A m = most[0];
    if constexpr (kWide) {
      // the largest in 64 bits: of a wave, then of the row
#pragma unroll
      for (int step = 1; step < kWave; step *= 2) top = fmax(top, __shfl_xor(top, step));
      if constexpr (WAVES > 1) {
        if (lane == 0) wides[wave] = top;
        __syncthreads();
        top = wides[0];
        for (int j = 1; j < WAVES; ++j) top = fmax(top, wides[j]);
      }
      m = top;
    }
    const bool finite = __builtin_bit_cast(uint32_t, most[0]) < 0x7F800000u;
    const bool zero = !(m > 0);
    // 127 / m would pass the range below 2^-121
    const bool tiny = !zero && most[0] < 0x1p-120f;
    const float inv = finite && !zero && !tiny ? 127.0f / most[0] : 0.0f;
    const Stream codes(static_cast<int8_t*>(a.y) + dense, static_cast<uint32_t>(a.width));
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      u32x2 v{0u, 0u};
      if (finite && !zero) {
        if constexpr (kWide) {
          float p[8];
          double wide[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            wide[i] = static_cast<double>(h[c][i]) * w[c][i];
            p[i] = h[c][i] * w[c][i];
          }
          v = codes_of(p, wide, m, inv, tiny);
        } else {
          v = codes_of(h[c], h[c], m, inv, tiny);
        }
      }
      E::template store_bytes<kNt>(codes, place(c), lane, v);
    }
    // of a row of zeros 0 also without eps, where size is infinite; m of 64 bits may have no place in 32
    if (lane == 0 && (WAVES == 1 || wave == 0)) {
      float scale;
      if constexpr (kWide)
        scale = static_cast<float>(static_cast<double>(size) * m / 127.0);
      else
        scale = size * m / 127.0f;
      a.scale[row] = !finite ? __builtin_nanf("") : zero ? 0.0f : scale;
    }
  }
}

struct BwdArgs {
  const void *dh, *dy, *h, *w;
  void *dx, *dres;
  float* parts;             // [workgroups][width]
  int64_t dhs[2], dys[2];
  Divisor rows;
  uint32_t total;
  int width;
  float eps;
  Drop drop;
};

// Lanes add dw up in registers over all their rows, waves that have rows of their own in
// LDS, and a second kernel adds the workgroups' sums, each in a fixed order.  32768 x 2048 bf16
// with dropout: 114 us with the second kernel's 4, 5.9 TB/s.
template <int DT, int WAVES, int CHUNKS, bool DROP>
__global__ __launch_bounds__(Group<WAVES>::kThreads) void rnorm_bwd_kernel(const BwdArgs a) {
  using T = typename Store<DT>::type;
  using G = Group<WAVES>;
  using E = Chunk<T>;
  __shared__ float parts[2][WAVES][2];
  __shared__ float sums[WAVES == 1 ? 4 : 1][WAVES == 1 ? CHUNKS * kWave * 8 : 1];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const auto place = [&](int c) __attribute__((always_inline)) { return (c * WAVES + (WAVES == 1 ? 0 : wave)) * kWaveElements; };
  const uint32_t bytes = static_cast<uint32_t>(a.width) * sizeof(T);
  // where 128 registers do not hold a row's four tensors, w and dh are read where they are used
  constexpr bool kLate = WAVES == 16 && CHUNKS == 4;
  float w[CHUNKS][8], dw[CHUNKS][8] = {};
  const Stream sw(a.w, bytes);
  if constexpr (!kLate)
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) E::template load<0>(sw, place(c), lane, w[c]);
  [[maybe_unused]] const Key key = DROP ? key_of(a.drop) : Key{};
  int turn = 0;
  for (uint32_t row = blockIdx.x * G::kRows + (WAVES == 1 ? wave : 0); row < a.total; row += gridDim.x * G::kRows, turn ^= 1) {
    const int64_t dense = static_cast<int64_t>(row) * a.width;
    const Stream sh(static_cast<const T*>(a.h) + dense, bytes), sy(row_of<T>(a.dy, row, a.rows, a.dys), bytes);
    const Stream sd(a.dh ? row_of<T>(a.dh, row, a.rows, a.dhs) : nullptr, a.dh ? bytes : 0);       // none: zeros
    float h[CHUNKS][8], g[CHUNKS][8], d[CHUNKS][8];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      E::template load<kNt>(sh, place(c), lane, h[c]);
      E::template load<kNt>(sy, place(c), lane, g[c]);
      if constexpr (!kLate) E::template load<kNt>(sd, place(c), lane, d[c]);
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      if constexpr (kLate) E::template load<0>(sw, place(c), lane, w[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum[0] += h[c][i] * h[c][i];
        sum[1] += g[c][i] * w[c][i] * h[c][i];
      }
    }
    over_row<WAVES>(sum, parts[turn], Add());
    const float r = 1.0f / sqrtf(sum[0] / a.width + a.eps);
    const float mean = sum[1] * r / a.width;              // of g h r
    const Stream dx(static_cast<T*>(a.dx) + dense, bytes), dres(static_cast<T*>(a.dres) + dense, a.dres ? bytes : 0);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      if constexpr (kLate) {
        E::template load<0>(sw, place(c), lane, w[c]);
        E::template load<kNt>(sd, place(c), lane, d[c]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = h[c][i] * r;
        dw[c][i] += g[c][i] * u;
        d[c][i] += r * (g[c][i] * w[c][i] - u * mean);
      }
      if constexpr (DROP) {
        E::template store<kNt>(dres, place(c), lane, d[c]);
        drop<T>(a.drop, key, static_cast<uint64_t>((dense + place(c)) / 8), lane, d[c]);
      }
      E::template store<kNt>(dx, place(c), lane, d[c]);
    }
  }
  const Stream out(a.parts + static_cast<int64_t>(blockIdx.x) * a.width, static_cast<uint32_t>(a.width) * 4);
  if constexpr (WAVES > 1) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) E::template store_floats<0>(out, place(c), lane, dw[c]);
  } else {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[wave][(c * 8 + i) * kWave + lane] = dw[c][i];
    __syncthreads();
#pragma unroll
    for (int c = wave; c < CHUNKS; c += 4) {
      float s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = (c * 8 + i) * kWave + lane;
        s[i] = (sums[0][at] + sums[1][at]) + (sums[2][at] + sums[3][at]);
      }
      E::template store_floats<0>(out, place(c), lane, s);
    }
  }
}

// The sums of the workgroups' rows of `width` floats: a workgroup takes 32 columns, a line of
// each row, 32 sums of every 32nd row each, then adds those in pairs.  (Eight columns by 128
// sums fetch every line four times, on as many XCDs: 8192 x 8192 bf16 with both kernels 126 us,
// so 118.)
constexpr int kColumns = 32, kRows = 32;
template <int DT>
__global__ __launch_bounds__(kColumns* kRows) void rnorm_sum_kernel(const float* parts, int rows, int width, void* dw) {
  __shared__ float sums[kRows][kColumns];
  const int at = threadIdx.x % kColumns, col = blockIdx.x * kColumns + at, row = threadIdx.x / kColumns;
  float sum = 0.0f;
  if (col < width)
#pragma unroll 8
    for (int r = row; r < rows; r += kRows) sum += parts[static_cast<int64_t>(r) * width + col];
  sums[row][at] = sum;
  for (int n = kRows / 2; n > 0; n /= 2) {
    __syncthreads();
    if (row < n) sums[row][at] += sums[row + n][at];
  }
  if (row == 0 && col < width) static_cast<typename Store<DT>::type*>(dw)[col] = static_cast<typename Store<DT>::type>(sums[0][at]);
}

// ---------------------------------------------------------------- host side
int check(const fewbit_rnorm* a) {
  if (!a) return FEWBIT_E_NULL;
  if (a->dtype < FEWBIT_F32 || a->dtype > FEWBIT_BF16) return FEWBIT_E_DTYPE;
  if ((a->dw_dtype != FEWBIT_F32 && a->dw_dtype != a->dtype) || a->outer < 0 || a->rows < 0) return FEWBIT_E_INVALID;
  if (a->width < 8 || a->width % 8 != 0 || a->width > FEWBIT_RNORM_MOST) return FEWBIT_E_INVALID;
  if (!(a->eps >= 0.0f && std::isfinite(a->eps))) return FEWBIT_E_INVALID;
  // rows are counted in 31 bits
  if (a->rows >= int64_t{1} << 31 || a->outer >= int64_t{1} << 31) return FEWBIT_E_INVALID;
  if (a->rows > 0 && a->outer > (((int64_t{1} << 31) - 1) / a->rows)) return FEWBIT_E_INVALID;
  Drop d;
  return drop_of(a->drop, d);
}

bool nothing(const fewbit_rnorm* a) { return a->outer == 0 || a->rows == 0; }
uint32_t total_of(const fewbit_rnorm* a) { return static_cast<uint32_t>(a->outer * a->rows); }

bool strides_fit(const fewbit_rnorm* a, const int64_t (&s)[2]) {
  const int64_t per = a->dtype == FEWBIT_F32 ? 4 : 8;
  return s[0] % per == 0 && s[1] % per == 0;
}

// Waves of a row and chunks of a lane.  Many rows take as few waves as hold them: a row of one
// needs no barrier (32768 rows of 8192 in 8 bits: four waves 126 us, 16 315).  Few rows take more,
// so that the loads of one are shorter in a row (64 rows of 8192: 16 waves 4.9 us, four 5.6).
struct Shape {
  int waves, chunks;
};
Shape shape_of(int width, bool few) {
  const int chunks = (width / 8 + kWave - 1) / kWave;       // of a wave
  const int waves = few ? (chunks <= 1 ? 1 : chunks <= 4 ? 4 : 16) : (chunks <= 4 ? 1 : chunks <= 16 ? 4 : 16);
  const int each = (chunks + waves - 1) / waves;
  return {waves, each <= 1 ? 1 : each <= 2 ? 2 : 4};
}

// Calls f with types that hold the shape.
template <int W, int C>
struct At {
  static constexpr int kWaves = W, kChunks = C;
};
template <class F>
hipError_t at_shape(Shape s, F f) {
  switch (s.waves * 8 + s.chunks) {
    case 9: return f(At<1, 1>());
    case 10: return f(At<1, 2>());
    case 12: return f(At<1, 4>());
    case 33: return f(At<4, 1>());
    case 34: return f(At<4, 2>());
    case 36: return f(At<4, 4>());
    case 129: return f(At<16, 1>());
    case 130: return f(At<16, 2>());
    default: return f(At<16, 4>());
  }
}

bool few_rows(const fewbit_rnorm* a) { return static_cast<int64_t>(total_of(a)) < 4 * device_cus(); }

template <int DT, Out OUT, bool DROP>
hipError_t start_fwd(const fewbit_rnorm* a, const FwdArgs& r, hipStream_t s) {
  return at_shape(shape_of(a->width, few_rows(a)), [&](auto at) {
    using S = decltype(at);
    using G = Group<S::kWaves>;
    return launch(rnorm_fwd_kernel<DT, S::kWaves, S::kChunks, OUT, DROP>, dim3((r.total + G::kRows - 1) / G::kRows), G::kThreads, s, r);
  });
}
template <int DT>
hipError_t start_out(const fewbit_rnorm* a, const FwdArgs& r, Out out, hipStream_t s) {
  if (out == kNorm8) return start_fwd<DT, kNorm8, false>(a, r, s);
  if (out == kRows8) return start_fwd<DT, kRows8, false>(a, r, s);
  return r.drop.border ? start_fwd<DT, kNorm, true>(a, r, s) : start_fwd<DT, kNorm, false>(a, r, s);
}

int forward(const char* where, const fewbit_rnorm* a, const void* x, const void* residual, const void* w, void* h, void* y, float* scale, Out out,
            void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  FwdArgs r{};
  if (out != kRows8) drop_of(a->drop, r.drop);
  if (out == kNorm8 && a->drop.p != 0.0) return FEWBIT_E_INVALID;
  if (nothing(a)) return FEWBIT_OK;
  const bool sums = out != kRows8 && (residual || r.drop.border > 0);
  if (!x || !y || (out != kRows8 && !w) || (out != kNorm && !scale) || (sums && !h)) return FEWBIT_E_NULL;
  if (misaligned(x) || misaligned(residual) || misaligned(w) || misaligned(h) || misaligned(y)) return FEWBIT_E_ALIGN;
  if (!strides_fit(a, a->x_stride) || (residual && !strides_fit(a, a->residual_stride))) return FEWBIT_E_ALIGN;
  r.x = x;
  r.res = residual;
  r.w = w;
  r.h = sums ? h : nullptr;
  r.y = y;
  r.scale = scale;
  for (int i = 0; i < 2; ++i) {
    r.xs[i] = a->x_stride[i];
    r.rs[i] = a->residual_stride[i];
  }
  r.rows = divisor(static_cast<int>(a->rows));
  r.total = total_of(a);
  r.width = a->width;
  r.eps = a->eps;
  const Shape shape = shape_of(a->width, few_rows(a));
  const int64_t groups = shape.waves == 1 ? (static_cast<int64_t>(r.total) + 3) / 4 : r.total;
  if (!fits_launch(groups, kWave * (shape.waves == 1 ? 4 : shape.waves))) return FEWBIT_E_INVALID;
  rc = check_stream_device(static_cast<hipStream_t>(stream));
  if (rc != FEWBIT_OK) return rc;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return launch_status(where, a->dtype == FEWBIT_F32   ? start_out<FEWBIT_F32>(a, r, out, s)
                              : a->dtype == FEWBIT_F16 ? start_out<FEWBIT_F16>(a, r, out, s)
                                                       : start_out<FEWBIT_BF16>(a, r, out, s));
}

// Workgroups of the backward, each of which leaves a row for the second kernel: two a CU, one
// where 16 waves hold a row.  (32768 x 2048 bf16 with dropout: 116 us, with one a CU 125, three
// 121, five 131.  The next row's loads ahead of a row's work, in registers: 115 to 120.)
int64_t groups_of(const fewbit_rnorm* a) {
  const Shape s = shape_of(a->width, few_rows(a));
  const int64_t rows = s.waves == 1 ? (static_cast<int64_t>(total_of(a)) + 3) / 4 : total_of(a);
  return std::min<int64_t>(rows, device_cus() * (s.waves == 16 ? 1 : 2));
}

template <int DT, bool DROP>
hipError_t start_bwd(const fewbit_rnorm* a, const BwdArgs& r, hipStream_t s) {
  return at_shape(shape_of(a->width, few_rows(a)), [&](auto at) {
    using S = decltype(at);
    return launch(rnorm_bwd_kernel<DT, S::kWaves, S::kChunks, DROP>, dim3(static_cast<unsigned>(groups_of(a))), Group<S::kWaves>::kThreads, s, r);
  });
}
template <int DT>
hipError_t start_back(const fewbit_rnorm* a, const BwdArgs& r, hipStream_t s) {
  return r.drop.border ? start_bwd<DT, true>(a, r, s) : start_bwd<DT, false>(a, r, s);
}

int64_t drop_groups(int64_t n) {
  constexpr int64_t kPer = int64_t{8} * kDropBlocks * kDropThreads;
  return (n + kPer - 1) / kPer;
}
template <int DT>
hipError_t start_drop(const void* x, void* y, int64_t n, const Drop& d, hipStream_t s) {
  return launch(drop_kernel<DT>, dim3(static_cast<unsigned>(drop_groups(n))), kDropThreads, s, x, y, n, d);
}

}  // namespace

extern "C" int fewbit_dropout(const fewbit_drop* d, int32_t dtype, int64_t n, const void* x, void* y, void* stream) {
  if (!d) return FEWBIT_E_NULL;
  if (dtype < FEWBIT_F32 || dtype > FEWBIT_BF16) return FEWBIT_E_DTYPE;
  Drop r{};
  int rc = drop_of(*d, r);
  if (rc != FEWBIT_OK) return rc;
  if (n < 0 || n >= int64_t{1} << 37 || !fits_launch(drop_groups(n), kDropThreads)) return FEWBIT_E_INVALID;
  if (n == 0) return FEWBIT_OK;
  if (!x || !y) return FEWBIT_E_NULL;
  if (misaligned(x) || misaligned(y)) return FEWBIT_E_ALIGN;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  rc = check_stream_device(s);
  if (rc != FEWBIT_OK) return rc;
  return launch_status("fewbit_dropout", dtype == FEWBIT_F32   ? start_drop<FEWBIT_F32>(x, y, n, r, s)
                                         : dtype == FEWBIT_F16 ? start_drop<FEWBIT_F16>(x, y, n, r, s)
                                                               : start_drop<FEWBIT_BF16>(x, y, n, r, s));
}

extern "C" int fewbit_rnorm_fwd(const fewbit_rnorm* a, const void* x, const void* residual, const void* w, void* h, void* y, void* stream) {
  return forward("fewbit_rnorm_fwd", a, x, residual, w, h, y, nullptr, kNorm, stream);
}

extern "C" int fewbit_rnorm_int8(const fewbit_rnorm* a, const void* x, const void* residual, const void* w, void* h, int8_t* codes, float* scale,
                                 void* stream) {
  return forward("fewbit_rnorm_int8", a, x, residual, w, h, codes, scale, kNorm8, stream);
}

extern "C" int fewbit_rows8(const fewbit_rnorm* a, const void* x, int8_t* codes, float* scale, void* stream) {
  return forward("fewbit_rows8", a, x, nullptr, nullptr, nullptr, codes, scale, kRows8, stream);
}

extern "C" int64_t fewbit_rnorm_workspace(const fewbit_rnorm* a) {
  const int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  return nothing(a) ? 0 : groups_of(a) * a->width * static_cast<int64_t>(sizeof(float));
}

extern "C" int fewbit_rnorm_bwd(const fewbit_rnorm* a, const void* dh, const void* dy, const void* h, const void* w, void* dx, void* dresidual,
                                void* dw, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  BwdArgs r{};
  drop_of(a->drop, r.drop);
  if (dresidual && r.drop.border == 0) return FEWBIT_E_INVALID;
  if (!dw) return FEWBIT_E_NULL;
  const bool none = nothing(a);             // no rows: the weight's gradient is 0
  int64_t groups = 0;
  if (!none) {
    if (!dy || !h || !w || !dx || !workspace) return FEWBIT_E_NULL;
    if (misaligned(dh) || misaligned(dy) || misaligned(h) || misaligned(w) || misaligned(dx) || misaligned(dresidual) || misaligned(workspace))
      return FEWBIT_E_ALIGN;
    if (!strides_fit(a, a->dy_stride) || (dh && !strides_fit(a, a->dh_stride))) return FEWBIT_E_ALIGN;
    if (workspace_bytes < fewbit_rnorm_workspace(a)) return FEWBIT_E_INVALID;
    groups = groups_of(a);
  }
  const hipStream_t s = static_cast<hipStream_t>(stream);
  rc = check_stream_device(s);
  if (rc != FEWBIT_OK) return rc;
  if (!none) {
    r.dh = dh;
    r.dy = dy;
    r.h = h;
    r.w = w;
    r.dx = dx;
    r.dres = dresidual;
    r.parts = static_cast<float*>(workspace);
    for (int i = 0; i < 2; ++i) {
      r.dhs[i] = a->dh_stride[i];
      r.dys[i] = a->dy_stride[i];
    }
    r.rows = divisor(static_cast<int>(a->rows));
    r.total = total_of(a);
    r.width = a->width;
    r.eps = a->eps;
    rc = launch_status("fewbit_rnorm_bwd", a->dtype == FEWBIT_F32   ? start_back<FEWBIT_F32>(a, r, s)
                                           : a->dtype == FEWBIT_F16 ? start_back<FEWBIT_F16>(a, r, s)
                                                                    : start_back<FEWBIT_BF16>(a, r, s));
    if (rc != FEWBIT_OK) return rc;
  }
  const auto sum = a->dw_dtype == FEWBIT_F32 ? rnorm_sum_kernel<FEWBIT_F32> : a->dw_dtype == FEWBIT_F16 ? rnorm_sum_kernel<FEWBIT_F16> : rnorm_sum_kernel<FEWBIT_BF16>;
  return launch_status("fewbit_rnorm_bwd", launch(sum, dim3((a->width + kColumns - 1) / kColumns), kColumns * kRows, s,
                                                  static_cast<const float*>(workspace), static_cast<int>(groups), a->width, dw));
}
