// mm8.hip -- product of tokens and weights in 8-bit integers, with a scale per token and
// per channel, bias and activation in the epilogue.
//
// Formulas in fewbit_residual.h.  Few tokens are bound by the weights' bytes, many by the
// matrix instructions (and the power that they draw: 32768 x 8192 by 2048 takes 400 us in a loop
// over the same codes, 2.7 POP/s, and 435 over several of full range).  The matrix instruction takes 16 channels by 16 tokens by
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
  Divisor group;            // tiles along the channels times kGroup
  uint32_t tiles, tiles_m;
  int* parts;               // sums of shares of the width [shares][rows][pitch], or NULL
  int64_t pitch;
  int each;                 // steps of a share
};

// Which tile a workgroup takes: consecutive workgroups go to the 8 XCDs in turn, so each XCD
// has a run of tiles of its own; a run goes through kGroup rows of tiles at a time, channels
// last, so that what runs together shares both operands in the XCD's L2.
constexpr int kXcds = 8, kGroup = 8;
struct Tile {
  int m, n;
};
__device__ __forceinline__ Tile tile_of(const Args& a, uint32_t block) {
  const uint32_t per = a.tiles / kXcds, more = a.tiles % kXcds, xcd = block % kXcds;
  const int at = static_cast<int>(xcd * per + min(xcd, more) + block / kXcds);
  const int g = a.group.divide(at), in = at - g * static_cast<int>(a.group.n);
  const int rows = min(kGroup, static_cast<int>(a.tiles_m) - g * kGroup);        // fewer in the last
  const int n = in / rows;
  return {g * kGroup + in - n * rows, n};
}

enum { kLinear = 0, kGelu = 1, kSilu = 2 };

// In fp32 whatever the result is stored as, so that half a step of that type is all it is off by:
// the fits of GELU that the few-bit forwards take for 16-bit results (bf16 1.9e-4 of the tail) put
// results on the other side of a border here and there.  It costs nothing that shows but in large
// products: 32768 x 2048 by 8192 bf16 550 us, with the fit for bf16 544.
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == kGelu) return Act<FEWBIT_F32, FEWBIT_GELU>::f(z);
  if constexpr (ACT == kSilu) return Act<FEWBIT_F32, FEWBIT_SILU>::f(z);
  return z;
}

// A result from its sum.  The sum meets one scale after the other: the product of both may pass
// fp32's range at either end where the result does not.
template <int ACT>
__device__ __forceinline__ float finished(int sum, float xs, float ws, float bias) {
  return activate<ACT>(static_cast<float>(sum) * xs * ws + bias);
}

// Rows from a matrix of codes into LDS, 128 bytes of each, by buffer loads that go there
// directly: a wave's load brings 8 rows of 8 chunks of 16 bytes.  Chunk c of row r lies at
// c ^ (r / 2 % 8), so that 16 lanes that read a chunk of 16 rows meet 64 different banks.
// What lies past the rows or the width reads as zeros.
constexpr int kStep = 128;            // bytes of a row that a stage holds

template <int ROWS, int WAVES>
struct Stage {
  static constexpr int kLoads = ROWS / 8 / WAVES;
  static_assert(WAVES % 2 == 0, "a wave's loads are whole swizzles apart");
  uint32_t offset[kLoads];
  int chunk;

  __device__ __forceinline__ Stage(int wave, int lane, uint32_t stride) {
    chunk = ((lane % 8) ^ ((wave * 8 + lane / 8) / 2 % 8)) * 16;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) offset[j] = ((j * WAVES + wave) * 8 + lane / 8) * stride + chunk;
  }
  // The chunks past `left` bytes are not there.
  __device__ __forceinline__ void cut(int left) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      if (chunk >= left) offset[j] = 0x80000000u;
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
  int width, wave;

  // Past the last step nothing is read and zeros are written.
  __device__ __forceinline__ void load(int step, int8_t* xt, int8_t* wt) {
    const int at = step * kStep, left = width - at;
    if (left < kStep) {
      sx.cut(left);
      sw.cut(left);
    }
    sx.load(x + at, left > 0 ? xb - at : 0, xt, wave);
    sw.load(w + at, left > 0 ? wb - at : 0, wt, wave);
  }
};

// Where a lane's 16 codes of row lane % 16 begin: chunk 4 half + lane / 16.
__device__ __forceinline__ int fragment(int half, int lane) { return lane % 16 * kStep + (((half * 4 + lane / 16) ^ (lane % 16 / 2)) * 16); }
__device__ __forceinline__ i32x4 codes(const int8_t* lds, int at, int row0) { return *reinterpret_cast<const i32x4*>(lds + at + row0 * kStep); }

// What the epilogue of a tile multiplies by and adds, on its way to LDS while the first
// stages are.  Channels and tokens past the end have zeros.
template <int BM, int BN>
struct Scales {
  float xs[BM], ws[BN], bias[BN];
};
struct Scale {
  float xs = 0.0f, ws = 0.0f, bias = 0.0f;
  template <class T>
  __device__ __forceinline__ void load(const Args& a, int64_t m, int64_t n) {
    if (m < a.rows) xs = a.xs[m];
    if (n < a.out) ws = a.ws[n];
    if (n < a.out && a.bias) bias = static_cast<float>(static_cast<const T*>(a.bias)[n]);
  }
  template <int BM, int BN>
  __device__ __forceinline__ void put(Scales<BM, BN>& s) const {
    if (threadIdx.x < BM) s.xs[threadIdx.x] = xs;
    if (threadIdx.x < BN) {
      s.ws[threadIdx.x] = ws;
      s.bias[threadIdx.x] = bias;
    }
  }
};

// Rows of WN elements from LDS to y, V bytes of a lane at a time.
template <class T, int WN, int ROWS, int V, bool KEEP>
__device__ __forceinline__ void store_rows(const int8_t* lds, T* y, int64_t out, int rows, int cols, int lane) {
  typedef T Piece __attribute__((ext_vector_type(V / sizeof(T))));
  constexpr int kPer = 16 / sizeof(T), kChunks = WN / kPer;       // of a chunk of 16 bytes
  constexpr int kEach = V / sizeof(T), kLanes = WN / kEach;       // elements of a lane, lanes of a row
#pragma unroll 8
  for (int at = lane; at < ROWS * kLanes; at += kWave) {
    const int r = at / kLanes, c = at % kLanes * kEach;
    const Piece v = *reinterpret_cast<const Piece*>(lds + (r * kChunks + (c / kPer ^ r / 2 % kChunks)) * 16 + c % kPer * sizeof(T));
    if (r < rows && c < cols) {
      if constexpr (KEEP)
        *reinterpret_cast<Piece*>(y + r * out + c) = v;
      else
        __builtin_nontemporal_store(v, reinterpret_cast<Piece*>(y + r * out + c));
    }
  }
}

// A wave's WM tokens by WN channels from its registers to y, through BYTES of LDS of its own, so
// that it stores whole runs of a row.  Element (r, c) lies in chunk c / kPer ^ r / 2 % kChunks of
// row r, so that lanes that write a chunk of 16 rows meet different banks (all but: of 16-bit
// results four cycles of conflicts are counted for every write of 8 bytes a lane).  KEEP: results
// stay in the caches, as those of tiles of 256 hardly would (32768 x 2048 by 8192 channels with
// GELU 628 us, past the caches 600, and with the channels' scales read once instead of for every
// 16 tokens 542, 550 with the fit for fp32).
template <int DT, int ACT, int WM, int WN, int BYTES, bool KEEP, int BM, int BN>
__device__ __forceinline__ void finish(const Args& a, const Scales<BM, BN>& s, int8_t* lds, int64_t m0, int64_t n0, int wm, int wn, int lane,
                                       const i32x4 (&acc)[WN / 16][WM / 16]) {
  using T = typename Store<DT>::type;
  typedef T V4 __attribute__((ext_vector_type(4)));
  constexpr int kPer = 16 / sizeof(T), kChunks = WN / kPer;       // elements of a chunk, chunks of a row
  constexpr int kRows = WM * kChunks * 16 <= BYTES ? WM : BYTES / (kChunks * 16) / 16 * 16;
  const int64_t m1 = m0 + wm, n1 = n0 + wn;
#pragma unroll
  for (int first = 0; first < WM; first += kRows) {
#pragma unroll
    for (int i = 0; i < WN / 16; ++i) {
      const int c = i * 16 + lane / 16 * 4;
      const f32x4 ws = *reinterpret_cast<const f32x4*>(s.ws + wn + c), bias = *reinterpret_cast<const f32x4*>(s.bias + wn + c);
#pragma unroll
      for (int j = first / 16; j < (first + kRows) / 16; ++j) {
        const int r = j * 16 - first + lane % 16;
        const float xs = s.xs[wm + j * 16 + lane % 16];
        V4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = static_cast<T>(finished<ACT>(acc[i][j][e], xs, ws[e], bias[e]));
        *reinterpret_cast<V4*>(lds + r * kChunks * 16 + ((c / kPer ^ r / 2 % kChunks) * 16) + c % kPer * sizeof(T)) = v;
      }
    }
    const int rows = static_cast<int>(min(static_cast<int64_t>(kRows), a.rows - m1 - first));
    const int cols = static_cast<int>(min(static_cast<int64_t>(WN), a.out - n1));
    T* y = static_cast<T*>(a.y) + (m1 + first) * a.out + n1;
    // by as many bytes as every row is aligned to
    const int aligned = static_cast<int>(a.out * sizeof(T) % 16);
    if (aligned == 0)
      store_rows<T, WN, kRows, 16, KEEP>(lds, y, a.out, rows, cols, lane);
    else if (aligned % 8 == 0)
      store_rows<T, WN, kRows, 8, KEEP>(lds, y, a.out, rows, cols, lane);
    else if (aligned % 4 == 0)
      store_rows<T, WN, kRows, 4, KEEP>(lds, y, a.out, rows, cols, lane);
    else
      store_rows<T, WN, kRows, sizeof(T), KEEP>(lds, y, a.out, rows, cols, lane);
  }
}

// A workgroup takes BM tokens by BN channels, a wave WM by WN of those, 128 codes at a step.
// While the matrix instructions work on half a step, the next half's operands come from LDS
// and the step after the next from memory.  Tokens' operands are replaced as soon as they
// have been used, channels' are held twice.  The two stages are arrays of their own, and each
// half of the loop knows which it reads: only then does a read of one not wait for the loads
// that are on their way to the other.
template <int WM, int WN>
struct Operands {
  i32x4 x[WM / 16], w[2][WN / 16];
  int xs[2], ws[2];         // places in a stage, of both halves

  // One half: `NEXT` is that of the operands that are brought meanwhile.
  template <int NEXT, int FROM, int TO>
  __device__ __forceinline__ void multiply(i32x4 (&acc)[WN / 16][WM / 16]) {
#pragma unroll
    for (int j = FROM; j < TO; ++j)
#pragma unroll
      for (int i = 0; i < WN / 16; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[1 - NEXT][i], x[j], acc[i][j], 0, 0, 0);
  }
  template <int NEXT, int FROM, int TO>
  __device__ __forceinline__ void read(const int8_t* xt, const int8_t* wt) {
#pragma unroll
    for (int j = FROM; j < TO; ++j) {
      x[j] = codes(xt, xs[NEXT], j * 16);
      if (j < WN / 16) w[NEXT][j] = codes(wt, ws[NEXT], j * 16);
    }
  }
  template <int NEXT, int FROM, int TO>
  __device__ __forceinline__ void both(const int8_t* xt, const int8_t* wt, i32x4 (&acc)[WN / 16][WM / 16]) {
    if constexpr (FROM < WM / 16) {
      multiply<NEXT, FROM, TO>(acc);
      read<NEXT, FROM, TO>(xt, wt);
      if constexpr (NEXT == 1) {
        // as written: left to itself the compiler gathers the reads before the barrier, which
        // then waits for them (32768 x 8192 by 2048: 2% slower)
        __builtin_amdgcn_sched_group_barrier(0x008 /* matrix */, (TO - FROM) * (WN / 16), 0);
        __builtin_amdgcn_sched_group_barrier(0x100 /* LDS reads */, FROM < WN / 16 ? 2 : 1, 0);
      }
      both<NEXT, TO, TO + 1>(xt, wt, acc);
    }
  }
};

// All loads but the wave's last `ON_THEIR_WAY` have arrived, of every wave.
template <int ON_THEIR_WAY>
__device__ __forceinline__ void arrived() {
  // vmcnt in bits 0-3 and 14-15, expcnt not waited for, lgkmcnt(0)
  __builtin_amdgcn_s_waitcnt((ON_THEIR_WAY & 15) | (ON_THEIR_WAY >> 4) << 14 | 0x0070);
  __builtin_amdgcn_s_barrier();
}

template <int DT, int ACT, int BM, int BN, int WM, int WN, int STAGES, bool SPLIT>
__global__ __launch_bounds__(BM / WM * (BN / WN) * kWave) void tile_kernel(const Args a) {
  constexpr int kWaves = BM / WM * (BN / WN);
  constexpr int kX = BM * kStep, kStage = (BM + BN) * kStep;
  constexpr int kLoads = kStage / (16 * kWave) / kWaves;          // of a stage, by each wave
  __shared__ __align__(16) int8_t s0[kStage];
  __shared__ __align__(16) int8_t s1[kStage];
  __shared__ __align__(16) int8_t s2[STAGES > 2 ? kStage : 16];
  __shared__ __align__(16) int8_t s3[STAGES > 3 ? kStage : 16];
  __shared__ __align__(16) Scales<BM, BN> scales;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  static_assert(WN <= WM && WM % 32 == 0, "operands of the channels come with the first tokens'");
  const Tile tile = tile_of(a, blockIdx.x);
  const int64_t m0 = static_cast<int64_t>(tile.m) * BM, n0 = static_cast<int64_t>(tile.n) * BN;
  const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
  // the share of the width
  const int begin = SPLIT ? blockIdx.y * a.each * kStep : 0, width = SPLIT ? min(a.each * kStep, a.width - begin) : a.width;
  const int8_t *x = a.x + m0 * a.x_stride + begin, *w = a.w + n0 * a.w_stride + begin;
  const uint32_t xb = static_cast<uint32_t>((min(a.rows - m0, static_cast<int64_t>(BM)) - 1) * a.x_stride + width);
  const uint32_t wb = static_cast<uint32_t>((min(a.out - n0, static_cast<int64_t>(BN)) - 1) * a.w_stride + width);
  Stage<BM, kWaves> sx(wave, lane, static_cast<uint32_t>(a.x_stride));
  Stage<BN, kWaves> sw(wave, lane, static_cast<uint32_t>(a.w_stride));
  const int steps = (width + kStep - 1) / kStep;
  Both<BM, BN, kWaves> stage{sx, sw, x, w, xb, wb, width, wave};
  i32x4 acc[WN / 16][WM / 16] = {};
  Operands<WM, WN> of;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    of.xs[half] = wm * kStep + fragment(half, lane);
    of.ws[half] = wn * kStep + fragment(half, lane);
  }
  Scale scale;
  if constexpr (!SPLIT)
    scale.template load<typename Store<DT>::type>(a, threadIdx.x < BM ? m0 + threadIdx.x : a.rows, threadIdx.x < BN ? n0 + threadIdx.x : a.out);
  stage.load(0, s0, s0 + kX);
  if constexpr (STAGES > 2) {
    stage.load(1, s1, s1 + kX);
    stage.load(2, s2, s2 + kX);
    if constexpr (STAGES > 3) stage.load(3, s3, s3 + kX);
  }
  if constexpr (!SPLIT) scale.put(scales);
  arrived<(STAGES > 2 ? (STAGES - 1) * kLoads : 0)>();
  if (STAGES == 2 && steps > 1) stage.load(1, s1, s1 + kX);
  of.template read<0, 0, WM / 16>(s0, s0 + kX);
  // a step whose operands' first half is there; past the last step what is read is not used
  const auto work = [&](int step, int8_t* here, const int8_t* next) __attribute__((always_inline)) {
    of.template both<1, 0, 1>(here, here + kX, acc);
    of.template multiply<0, 0, 2>(acc);
    arrived<(STAGES - 2) * kLoads>();       // the next stage; and none reads this one any more
    // (the wait counts loads, so with more than two stages they are issued past the end too)
    if (STAGES > 2 || step + STAGES < steps) stage.load(step + STAGES, here, here + kX);
    of.template read<0, 0, 2>(next, next + kX);
    of.template both<0, 2, 3>(next, next + kX, acc);
  };
  int step = 0;
  for (; step + STAGES <= steps; step += STAGES) {
    work(step, s0, s1);
    if constexpr (STAGES == 2) work(step + 1, s1, s0);
    if constexpr (STAGES > 2) work(step + 1, s1, s2);
    if constexpr (STAGES == 3) work(step + 2, s2, s0);
    if constexpr (STAGES > 3) work(step + 2, s2, s3);
    if constexpr (STAGES > 3) work(step + 3, s3, s0);
  }
  if (step < steps) work(step, s0, s1);
  if constexpr (STAGES > 2) {
    if (step + 1 < steps) work(step + 1, s1, s2);
    if constexpr (STAGES > 3) {
      if (step + 2 < steps) work(step + 2, s2, s3);
    }
  }
  arrived<0>();             // nothing is on its way to the stages any more, and none reads them
  if constexpr (SPLIT) {
    int* parts = a.parts + blockIdx.y * a.rows * a.pitch;
#pragma unroll
    for (int j = 0; j < WM / 16; ++j) {
      const int64_t m = m0 + wm + j * 16 + lane % 16;
#pragma unroll
      for (int i = 0; i < WN / 16; ++i) {
        const int64_t n = n0 + wn + i * 16 + lane / 16 * 4;
        if (m < a.rows && n < a.out) *reinterpret_cast<i32x4*>(parts + m * a.pitch + n) = acc[i][j];
      }
    }
  } else {
    // results leave through two stages: half the waves' through each
    constexpr int kOwn = kStage / (kWaves / 2), kBytes = 8192;       // (16384: 1 to 3% slower, for stores begin later)
    static_assert(kOwn >= kBytes, "the waves' shares of the stages");
    finish<DT, ACT, WM, WN, kBytes, BM < 256>(a, scales, (wave % 2 ? s1 : s0) + wave / 2 * kBytes, m0, n0, wm, wn, lane, acc);
  }
}

// Sums of the shares, and the epilogue: a lane takes four consecutive channels.
constexpr int kJoinThreads = 64;          // small workgroups, for many CUs
template <int DT, int ACT>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const Args a, int shares) {
  using T = typename Store<DT>::type;
  const uint32_t quads = static_cast<uint32_t>(a.pitch / 4);
  const uint32_t at = blockIdx.x * kJoinThreads + threadIdx.x, m = at / quads;
  if (m >= a.rows) return;
  const int64_t n = (at - m * quads) * 4;
  const int* parts = a.parts + m * a.pitch + n;
  const T* biases = static_cast<const T*>(a.bias);
  // everything is on its way before the first is waited for; a row's last channels are read again
  // past its end
  const float xs = a.xs[m];
  float ws[4], bias[4] = {};
#pragma unroll
  for (int e = 0; e < 4; ++e) ws[e] = a.ws[min(n + e, a.out - 1)];
  if (biases)
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = static_cast<float>(biases[min(n + e, a.out - 1)]);
  i32x4 sum = {};
#pragma unroll 8
  for (int i = 0; i < shares; ++i) sum += *reinterpret_cast<const i32x4*>(parts + i * a.rows * a.pitch);
  T* y = static_cast<T*>(a.y) + m * a.out + n;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.out) y[e] = static_cast<T>(finished<ACT>(sum[e], xs, ws[e], bias[e]));
}

// ---------------------------------------------------------------- few tokens
// Up to 16 / H tokens (one by 8192 x 2048 weights: 5.4 us, 3.1 TB/s; 2048 x 8192 with H = 2: 5.9,
// H = 1 7.7; eight or 16 waves a workgroup are slower everywhere): a workgroup takes 16 / H channels, and its waves share the width in runs
// of 128 codes of H places each, straight from memory to the matrix instructions' operands: row
// r of an operand is channel (or token) r % (16 / H) at place r / (16 / H), and of the result
// only what has both places alike is wanted.  With H > 1 few channels make as many workgroups
// as there are CUs.  Loads are whole lines of each channel; those of the next runs are on their
// way while the last ones are multiplied.  The waves' sums meet in LDS.
constexpr int kRun = 128, kFewWaves = 4;

template <int DT, int ACT, int H>
__global__ __launch_bounds__(kFewWaves* kWave) void few_kernel(const Args a) {
  using T = typename Store<DT>::type;
  constexpr int kRows = 16 / H, kDeep = 2, WAVES = kFewWaves;
  __shared__ __align__(16) int sums[WAVES][16][16];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kRows;
  const uint32_t xb = static_cast<uint32_t>((a.rows - 1) * a.x_stride + a.width);
  const uint32_t wb = static_cast<uint32_t>((min(a.out - n0, static_cast<int64_t>(kRows)) - 1) * a.w_stride + a.width);
  const Stream x(a.x, xb), w(a.w + n0 * a.w_stride, wb);
  const int row = lane % kRows, place = lane % 16 / kRows;
  const uint32_t xo = row * static_cast<uint32_t>(a.x_stride), wo = row * static_cast<uint32_t>(a.w_stride);
  const bool some = row < a.rows;
  struct Runs {
    i32x4 x[kDeep][2], w[kDeep][2];
  };
  const auto load = [&](Runs& r, int run) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int at = ((run + d * WAVES) * H + place) * kRun + lane / 16 * 32 + half * 16;
        const bool in = at < a.width;           // else nothing is read, and zeros are taken
        r.w[d][half] = __builtin_bit_cast(i32x4, w.template get<kNt, 16>(in ? wo + at : 0x80000000u));
        r.x[d][half] = __builtin_bit_cast(i32x4, x.template get<0, 16>(in && some ? xo + at : 0x80000000u));
      }
  };
  i32x4 acc = {};
  const auto multiply = [&](const Runs& r) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
#pragma unroll
      for (int half = 0; half < 2; ++half) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(r.w[d][half], r.x[d][half], acc, 0, 0, 0);
  };
  // runs past the width are loads of nothing
  constexpr int kEach = WAVES * kDeep;
  const int runs = (a.width + kRun * H - 1) / (kRun * H);
  Runs even, odd;
  load(even, wave);
  for (int run = wave; run < runs; run += 2 * kEach) {
    load(odd, run + kEach);
    multiply(even);
    load(even, run + 2 * kEach);
    multiply(odd);
  }
  *reinterpret_cast<i32x4*>(&sums[wave][lane % 16][lane / 16 * 4]) = acc;
  __syncthreads();
  if (threadIdx.x >= kRows * kRows) return;
  const int r = threadIdx.x / kRows, c = threadIdx.x % kRows;
  const int64_t n = n0 + c;
  if (r >= a.rows || n >= a.out) return;
  int sum = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i)
#pragma unroll
    for (int h = 0; h < H; ++h) sum += sums[i][h * kRows + r][h * kRows + c];
  const float bias = a.bias ? static_cast<float>(static_cast<const T*>(a.bias)[n]) : 0.0f;
  static_cast<T*>(a.y)[r * a.out + n] = static_cast<T>(finished<ACT>(sum, a.xs[r], a.ws[n], bias));
}

// ---------------------------------------------------------------- host side
// A tile's rows are reached by offsets of 31 bits.
static_assert(int64_t{255} * FEWBIT_MM8_STRIDE + 131056 < int64_t{1} << 31, "offsets of a tile's rows");

int check(const fewbit_mm8* a) {
  if (!a) return FEWBIT_E_NULL;
  if (a->dtype < FEWBIT_F32 || a->dtype > FEWBIT_BF16) return FEWBIT_E_DTYPE;
  if (a->act != FEWBIT_MM8_LINEAR && a->act != FEWBIT_GELU && a->act != FEWBIT_SILU) return FEWBIT_E_INVALID;
  if (a->reserved != 0 || a->rows < 0 || a->out < 0 || a->rows >= int64_t{1} << 31 || a->out >= int64_t{1} << 31) return FEWBIT_E_INVALID;
  if (a->width < 16 || a->width > 131056 || a->width % 16 != 0) return FEWBIT_E_INVALID;
  if (a->x_stride < 0 || a->w_stride < 0 || a->x_stride > FEWBIT_MM8_STRIDE || a->w_stride > FEWBIT_MM8_STRIDE) return FEWBIT_E_INVALID;
  return FEWBIT_OK;
}

bool nothing(const fewbit_mm8* a) { return a->rows == 0 || a->out == 0; }

// How a product is done.
struct Plan {
  enum Kind { kFew, kTile64, kTile128Alone, kTile128, kTile256 } kind;
  int places;               // few tokens: H
  int shares, each;         // of the width, and a share's steps
  int64_t tiles_m, tiles_n;
};

// What is fastest by the times that each kernel was seen to take: of a step of 128 codes, and
// of the rest, in us, with T workgroups on 256 CUs.
//   few tokens   16.8 M weights by one token 5.4 us, in tiles 6.3; 67 M 14.4 and 11.4; 32 M by
//                four 13.7 and 10.2; by 16 tokens 4.2 M 4.3 and 6.5, 16.8 M 6.5 to 10.4 and 6.2
//                to 8.6; 228 channels of 15280 codes by 13: 22 and, in shares, 8.4
//   64 x 64      0.2 a step with a workgroup a CU (64 x 8192 by 2048: 6.1 us; with two stages
//                instead of four 10.3), 0.38 with two
//   128 x 128    three stages, a workgroup a CU: 0.6 (2048 x 2048 by 2048: 13.5 us, 64 x 64
//                17, 256 x 256 25); two stages, two workgroups a CU: 1.1 for both
//   256 x 256    1.5 (32768 x 8192 by 2048: 405 us, 128 x 128 541, 64 x 64 822)
//   shares       the second kernel takes 3.5, and 8 bytes of each share's sums at 3 TB/s
//                (64 x 8192 by 2048 channels: one 14.4 us, four 10.4)
Plan plan_of(const fewbit_mm8* a) {
  const double cus = device_cus();
  const int steps = (a->width + kStep - 1) / kStep;
  const int64_t weights = a->out * a->width;
  Plan best{Plan::kFew, 1, 1, steps, 1, 1};
  if (a->rows <= 16 && weights <= (a->rows <= 2 ? 1 << 25 : a->rows <= 8 ? 1 << 24 : 1 << 23)) {
    while (best.places < 4 && a->rows <= 8 / best.places && a->out * best.places < 16 * cus) best.places *= 2;
    if (a->width <= 4096 * best.places) return best;
  }
  double least = 0.0;
  const auto offer = [&](Plan::Kind kind, int side, int shares, int each, double per_cu, double step, double rest) {
    const int64_t tm = (a->rows + side - 1) / side, tn = (a->out + side - 1) / side;
    const double turns = std::ceil(static_cast<double>(tm) * tn * shares / (per_cu * cus));
    const double time = turns * (step * each + rest) + (shares > 1 ? 3.5 + 8e-6 / 3.0 * shares * a->rows * a->out : 0.0);
    if (least != 0.0 && time >= least) return;
    least = time;
    best = {kind, 1, shares, each, tm, tn};
  };
  const auto fits = [&](int side, int shares) {      // a workgroup a CU
    return static_cast<double>((a->rows + side - 1) / side) * ((a->out + side - 1) / side) * shares <= cus;
  };
  offer(Plan::kTile256, 256, 1, steps, 1, 1.5, 6.0);
  if (fits(128, 1))
    offer(Plan::kTile128Alone, 128, 1, steps, 1, 0.6, 4.0);
  else
    offer(Plan::kTile128, 128, 1, steps, 2, 1.1, 5.0);
  for (int shares = 1; shares <= 8 && (shares == 1 || steps / shares >= 4); shares *= 2) {
    const int each = (steps + shares - 1) / shares, real = (steps + each - 1) / each;
    if (fits(64, real))
      offer(Plan::kTile64, 64, real, each, 1, 0.2, 3.0);
    else if (real == 1 || fits(64, (real + 1) / 2))
      offer(Plan::kTile64, 64, real, each, 2, 0.38, 3.0);
  }
  return best;
}

int64_t threads_of(const Plan& p) { return p.kind == Plan::kTile256 ? 512 : 256; }

// Channels of a row of the shares' sums: rows start at whole quads.
int64_t pitch_of(const fewbit_mm8* a) { return (a->out + 3) / 4 * 4; }

template <int DT, int ACT, int SIDE, int WM, int WN, int STAGES>
hipError_t start_tiles(const Args& r, const Plan& p, hipStream_t s) {
  constexpr int kThreads = SIDE / WM * (SIDE / WN) * kWave;
  if constexpr (SIDE == 64) {       // the tiles that shares are offered for
    if (p.shares > 1) {
      // the sums do not depend on the types and the activation
      const hipError_t e = launch(tile_kernel<FEWBIT_F32, kLinear, SIDE, SIDE, WM, WN, STAGES, true>, dim3(r.tiles, p.shares), kThreads, s, r);
      if (e != hipSuccess) return e;
      const int64_t quads = r.rows * (r.pitch / 4);
      return launch(join_kernel<DT, ACT>, dim3(static_cast<unsigned>((quads + kJoinThreads - 1) / kJoinThreads)), kJoinThreads, s, r, p.shares);
    }
  }
  return launch(tile_kernel<DT, ACT, SIDE, SIDE, WM, WN, STAGES, false>, dim3(r.tiles), kThreads, s, r);
}
template <int DT, int ACT, int H>
hipError_t start_few(const Args& r, hipStream_t s) {
  constexpr int64_t kCols = 16 / H;
  return launch(few_kernel<DT, ACT, H>, dim3(static_cast<unsigned>((r.out + kCols - 1) / kCols)), kFewWaves * kWave, s, r);
}
template <int DT, int ACT>
hipError_t start_act(const Args& r, const Plan& p, hipStream_t s) {
  switch (p.kind) {
    case Plan::kFew:
      return p.places == 1 ? start_few<DT, ACT, 1>(r, s) : p.places == 2 ? start_few<DT, ACT, 2>(r, s) : start_few<DT, ACT, 4>(r, s);
    case Plan::kTile64: return start_tiles<DT, ACT, 64, 32, 32, 4>(r, p, s);
    case Plan::kTile128Alone: return start_tiles<DT, ACT, 128, 64, 64, 3>(r, p, s);
    case Plan::kTile128: return start_tiles<DT, ACT, 128, 64, 64, 2>(r, p, s);
    default: return start_tiles<DT, ACT, 256, 128, 64, 2>(r, p, s);
  }
}
template <int DT>
hipError_t start_dt(const fewbit_mm8* a, const Args& r, const Plan& p, hipStream_t s) {
  return a->act == FEWBIT_GELU ? start_act<DT, kGelu>(r, p, s) : a->act == FEWBIT_SILU ? start_act<DT, kSilu>(r, p, s) : start_act<DT, kLinear>(r, p, s);
}

}  // namespace

extern "C" int64_t fewbit_mm8_workspace(const fewbit_mm8* a) {
  const int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  if (nothing(a)) return 0;
  const Plan p = plan_of(a);
  return p.shares > 1 ? p.shares * a->rows * pitch_of(a) * static_cast<int64_t>(sizeof(int)) : 0;
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
  const Plan p = plan_of(a);
  const int64_t need = fewbit_mm8_workspace(a);
  if (need > 0 && !workspace) return FEWBIT_E_NULL;
  if (workspace_bytes < need) return FEWBIT_E_INVALID;
  if (p.kind == Plan::kFew ? !fits_launch((a->out * p.places + 15) / 16, kFewWaves * kWave)
                           : p.tiles_n >= int64_t{1} << 28 || !fits_launch(p.tiles_n * p.tiles_m, threads_of(p)))
    return FEWBIT_E_INVALID;
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
  r.tiles = static_cast<uint32_t>(p.tiles_m * p.tiles_n);
  r.tiles_m = static_cast<uint32_t>(p.tiles_m);
  r.group = divisor(static_cast<int>(p.tiles_n * kGroup));
  r.parts = static_cast<int*>(workspace);
  r.pitch = pitch_of(a);
  r.each = p.each;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  rc = check_stream_device(s);
  if (rc != FEWBIT_OK) return rc;
  return launch_status("fewbit_mm8_fwd", a->dtype == FEWBIT_F32   ? start_dt<FEWBIT_F32>(a, r, p, s)
                                         : a->dtype == FEWBIT_F16 ? start_dt<FEWBIT_F16>(a, r, p, s)
                                                                  : start_dt<FEWBIT_BF16>(a, r, p, s));
}
