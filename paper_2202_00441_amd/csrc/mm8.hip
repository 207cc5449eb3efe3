// mm8.hip -- product of tokens and weights in 8-bit integers, with a scale per token and
// per channel, bias and activation in the epilogue.
//
// Formulas in fewbit_residual.h.  The matrix instruction takes 16 channels by 16 tokens by
// 64 bytes of both: its first operand holds, in lane l, 16 consecutive codes of channel l %
// 16, the second those of token l % 16, and a lane of the result has four consecutive
// channels of one token.  Which 64 codes an instruction takes does not matter as long as
// both operands agree.
#include <algorithm>

#include "activations.h"
#include "block.h"
#include "fewbit_residual.h"

namespace {

using namespace block;

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Args {
  const int8_t *x, *w;
  const float *xs, *ws;
  const void* bias;
  void* y;
  int64_t rows, out;
  int64_t x_stride, w_stride;
  int width;
  uint32_t tiles_n;         // tiles along the channels
};

enum { kLinear = 0, kGelu = 1, kSilu = 2 };

template <int DT, int ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == kGelu) return Act<DT, FEWBIT_GELU>::f(z);
  if constexpr (ACT == kSilu) return Act<DT, FEWBIT_SILU>::f(z);
  return z;
}

// Rows from a matrix of codes into LDS, 128 bytes of each, by buffer loads that go there
// directly: a wave's load brings 8 rows of 8 chunks of 16 bytes.  Chunk c of row r lies at
// c ^ (r / 2 % 8), so that 16 lanes that read a chunk of 16 rows meet 64 different banks.
// What lies past the rows or the width reads as zeros.
constexpr int kStep = 128;            // bytes of a row that a stage holds

template <int ROWS, int WAVES>
struct Stage {
  static constexpr int kLoads = ROWS / 8 / WAVES;
  uint32_t offset[kLoads];

  __device__ __forceinline__ Stage(int wave, int lane, uint32_t stride) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = (j * WAVES + wave) * 8 + lane / 8;
      offset[j] = row * stride + ((lane % 8) ^ (row / 2 % 8)) * 16;
    }
  }
  // The chunks past `left` bytes are not there.
  __device__ __forceinline__ void cut(int wave, int lane, int left) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = (j * WAVES + wave) * 8 + lane / 8;
      if (((lane % 8) ^ (row / 2 % 8)) * 16 >= left) offset[j] = 0x80000000u;
    }
  }
  __device__ __forceinline__ void load(const int8_t* base, uint32_t bytes, int8_t* lds, int wave) const {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(base), 0, static_cast<int>(bytes), 0x00020000);
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (j * WAVES + wave) * 8 * kStep), 16,
                                               offset[j], 0, 0, 0);
  }
};

// The same 128 codes of a tile's tokens and of its channels.
template <int BM, int BN, int WAVES>
struct Both {
  Stage<BM, WAVES> sx;
  Stage<BN, WAVES> sw;
  const int8_t *x, *w;
  uint32_t xb, wb;
  int width, wave, lane;

  __device__ __forceinline__ void load(int step, int8_t* xt, int8_t* wt) {
    const int at = step * kStep, left = width - at;
    if (left < kStep) {
      sx.cut(wave, lane, left);
      sw.cut(wave, lane, left);
    }
    sx.load(x + at, xb - at, xt, wave);
    sw.load(w + at, wb - at, wt, wave);
  }
};

// 16 codes of row `row0 + lane % 16`: chunk 4 half + lane / 16.
__device__ __forceinline__ i32x4 fragment(const int8_t* lds, int row0, int half, int lane) {
  const int row = row0 + lane % 16;
  return *reinterpret_cast<const i32x4*>(lds + row * kStep + (((half * 4 + lane / 16) ^ (row / 2 % 8)) * 16));
}

// Four consecutive channels from n on of token m.
template <int DT, int ACT>
__device__ __forceinline__ void finish(const Args& a, int64_t m, int64_t n, i32x4 sum) {
  using T = typename Store<DT>::type;
  if (m >= a.rows || n >= a.out) return;
  const float xs = a.xs[m];
  T* y = static_cast<T*>(a.y) + m * a.out + n;
  const T* bias = static_cast<const T*>(a.bias);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n + i >= a.out) break;
    float z = static_cast<float>(sum[i]) * (xs * a.ws[n + i]);
    if (bias) z += static_cast<float>(bias[n + i]);
    y[i] = static_cast<T>(activate<DT, ACT>(z));
  }
}

// A workgroup takes BM tokens by BN channels, a wave WM by WN of those; the stage of the
// next 128 codes is on its way while one is worked on.
template <int DT, int ACT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(BM / WM * (BN / WN) * kWave) void tile_kernel(const Args a) {
  constexpr int kWaves = BM / WM * (BN / WN);
  __shared__ __align__(16) int8_t xt[2][BM * kStep];
  __shared__ __align__(16) int8_t wt[2][BN * kStep];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / a.tiles_n) * BM, n0 = static_cast<int64_t>(blockIdx.x % a.tiles_n) * BN;
  const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
  const int8_t *x = a.x + m0 * a.x_stride, *w = a.w + n0 * a.w_stride;
  const uint32_t xb = static_cast<uint32_t>((min(a.rows - m0, static_cast<int64_t>(BM)) - 1) * a.x_stride + a.width);
  const uint32_t wb = static_cast<uint32_t>((min(a.out - n0, static_cast<int64_t>(BN)) - 1) * a.w_stride + a.width);
  Stage<BM, kWaves> sx(wave, lane, static_cast<uint32_t>(a.x_stride));
  Stage<BN, kWaves> sw(wave, lane, static_cast<uint32_t>(a.w_stride));
  const int steps = (a.width + kStep - 1) / kStep;
  Both<BM, BN, kWaves> stage{sx, sw, x, w, xb, wb, a.width, wave, lane};
  i32x4 acc[WN / 16][WM / 16] = {};
  stage.load(0, xt[0], wt[0]);
  for (int step = 0; step < steps; ++step) {
    __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0): this step's stage, issued a step ago
    __syncthreads();                        // of all waves; and none reads the other any more
    if (step + 1 < steps) stage.load(step + 1, xt[(step + 1) % 2], wt[(step + 1) % 2]);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      i32x4 fx[WM / 16], fw[WN / 16];
#pragma unroll
      for (int i = 0; i < WM / 16; ++i) fx[i] = fragment(xt[step % 2], wm + i * 16, half, lane);
#pragma unroll
      for (int i = 0; i < WN / 16; ++i) fw[i] = fragment(wt[step % 2], wn + i * 16, half, lane);
#pragma unroll
      for (int i = 0; i < WN / 16; ++i)
#pragma unroll
        for (int j = 0; j < WM / 16; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int i = 0; i < WN / 16; ++i)
#pragma unroll
    for (int j = 0; j < WM / 16; ++j) finish<DT, ACT>(a, m0 + wm + j * 16 + lane % 16, n0 + wn + i * 16 + lane / 16 * 4, acc[i][j]);
}

// ---------------------------------------------------------------- host side
constexpr int64_t kMostStride = int64_t{1} << 22;      // a tile's rows are reached by offsets of 31 bits

int check(const fewbit_mm8* a) {
  if (!a) return FEWBIT_E_NULL;
  if (a->dtype < FEWBIT_F32 || a->dtype > FEWBIT_BF16) return FEWBIT_E_DTYPE;
  if (a->act != FEWBIT_MM8_LINEAR && a->act != FEWBIT_GELU && a->act != FEWBIT_SILU) return FEWBIT_E_INVALID;
  if (a->reserved != 0 || a->rows < 0 || a->out < 0 || a->rows >= int64_t{1} << 31 || a->out >= int64_t{1} << 31) return FEWBIT_E_INVALID;
  if (a->width < 16 || a->width > 131056 || a->width % 16 != 0) return FEWBIT_E_INVALID;
  if (a->x_stride < 0 || a->w_stride < 0 || a->x_stride > kMostStride || a->w_stride > kMostStride) return FEWBIT_E_INVALID;
  return FEWBIT_OK;
}

bool nothing(const fewbit_mm8* a) { return a->rows == 0 || a->out == 0; }

template <int DT, int ACT>
hipError_t start_act(const Args& r, hipStream_t s) {
  constexpr int kM = 128, kN = 128;
  Args t = r;
  t.tiles_n = static_cast<uint32_t>((r.out + kN - 1) / kN);
  const int64_t tiles = t.tiles_n * ((r.rows + kM - 1) / kM);
  if (!fits_launch(tiles, 256)) return hipErrorInvalidConfiguration;
  return launch(tile_kernel<DT, ACT, kM, kN, 64, 64>, dim3(static_cast<unsigned>(tiles)), 256, s, t);
}
template <int DT>
hipError_t start_dt(const fewbit_mm8* a, const Args& r, hipStream_t s) {
  return a->act == FEWBIT_GELU ? start_act<DT, kGelu>(r, s) : a->act == FEWBIT_SILU ? start_act<DT, kSilu>(r, s) : start_act<DT, kLinear>(r, s);
}

}  // namespace

extern "C" int64_t fewbit_mm8_workspace(const fewbit_mm8* a) {
  const int rc = check(a);
  return rc != FEWBIT_OK ? rc : 0;
}

extern "C" int fewbit_mm8_fwd(const fewbit_mm8* a, const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale, const void* bias,
                              void* y, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  if (nothing(a)) return FEWBIT_OK;
  if (!x || !x_scale || !w || !w_scale || !y) return FEWBIT_E_NULL;
  if (misaligned(x) || misaligned(w) || misaligned(x_scale) || misaligned(w_scale) || misaligned(bias) || misaligned(y) || misaligned(workspace))
    return FEWBIT_E_ALIGN;
  if (a->x_stride % 16 != 0 || a->w_stride % 16 != 0) return FEWBIT_E_ALIGN;
  if (workspace_bytes < fewbit_mm8_workspace(a)) return FEWBIT_E_INVALID;
  Args r{};
  r.x = x;
  r.w = w;
  r.xs = x_scale;
  r.ws = w_scale;
  r.bias = bias;
  r.y = y;
  r.rows = a->rows;
  r.out = a->out;
  r.x_stride = a->x_stride;
  r.w_stride = a->w_stride;
  r.width = a->width;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  rc = check_stream_device(s);
  if (rc != FEWBIT_OK) return rc;
  return launch_status("fewbit_mm8_fwd", a->dtype == FEWBIT_F32   ? start_dt<FEWBIT_F32>(a, r, s)
                                         : a->dtype == FEWBIT_F16 ? start_dt<FEWBIT_F16>(a, r, s)
                                                                  : start_dt<FEWBIT_BF16>(a, r, s));
}
