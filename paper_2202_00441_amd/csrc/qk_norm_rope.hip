// qk_norm_rope.hip -- RMS norm of every query and key head and its rotary
// position in one pass, and the gradients.
//
// Formulas in fewbit_block.h.  Bound by HBM: the forward reads and writes each
// element once; the backward reads the input and the incoming gradient and
// writes the gradient, and recomputes the norm instead of keeping it.
//
// A row (one head of one token) is held by a group of 4, 8 or 16 lanes, 16 elements
// each: two 16-byte chunks that hold both elements of eight rotated pairs, so that
// neither the rotation nor the tables' angles cross lanes, and the row's sums take two
// to four cross-lane steps.  A group takes several heads of one token at once: the
// token's angles are read once, and the rows are all on their way before the first is
// worked on.
//
// Backward: with g the incoming gradient turned back, x the input, r = 1 /
// sqrt(mean(x^2) + eps) and u = x r,
//   dw = sum over rows of g u,   dx = r (g w - u mean(g w u)).
// Lanes add dw up in registers over all their rows, waves across lanes, workgroups in LDS,
// and a second kernel adds the workgroups' sums, each in a fixed order.
#include <algorithm>

#include "block.h"

namespace {

using namespace block;

constexpr int kThreads = 256;
constexpr int kN = 16;          // elements of a lane

struct Side {
  const void* x;
  const void* w;
  const void* dy;       // backward
  void* y;              // forward: output; backward: gradient
  int64_t xs[3], ds[3];
  int heads;
  Divisor shares;       // groups of a token
  uint32_t units;       // groups of all tokens
};

struct Args {
  Side s[2];
  const float *cos, *sin;
  const int64_t* pos;
  int64_t ps[2];
  int64_t table_rows;
  Divisor tokens;
  int d, rot;
  uint32_t first_k;     // the first workgroup of the keys
  float eps;
  float* parts;         // backward: [workgroups][head_dim]
};

// Where a lane's two chunks of eight elements begin in a row.
struct Chunks {
  int a, b;
  bool some, turned;
};
template <bool INTER>
__device__ __forceinline__ Chunks chunks_of(int lane, int d, int rot) {
  if (INTER) return {16 * lane, 16 * lane + 8, 16 * lane < d, 16 * lane < rot};
  const int half = rot / 2;
  if (8 * lane < half) return {8 * lane, 8 * lane + half, true, true};
  const int at = rot + 16 * lane - 2 * half;            // past the rotated part
  return {at, at + 8, at < d, false};
}

// x[0..7], x[8..15] are a lane's chunks; pair j is (x[j], x[8 + j]), or, of
// adjacent elements, (x[2j], x[2j + 1]).
template <bool INTER>
__device__ __forceinline__ void turn(float (&x)[kN], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float &a = x[INTER ? 2 * j : j], &b = x[INTER ? 2 * j + 1 : 8 + j];
    const float u = a * c[j] - b * s[j];
    b = b * c[j] + a * s[j];
    a = u;
  }
}

// A lane's part of a row as it lies in memory, and as fp32.
template <class T>
struct Raw {
  static constexpr int kVecs = 8 * sizeof(T) / 16;      // 16-byte accesses of a chunk
  typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
  V v[2 * kVecs];

  __device__ __forceinline__ void load(const T* row, const Chunks& at) {
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      v[j] = __builtin_nontemporal_load(reinterpret_cast<const V*>(row + at.a) + j);
      v[kVecs + j] = __builtin_nontemporal_load(reinterpret_cast<const V*>(row + at.b) + j);
    }
  }
  __device__ __forceinline__ void get(float (&x)[kN]) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = static_cast<float>(v[i / (8 / kVecs)][i % (8 / kVecs)]);
  }
};
template <class T>
__device__ __forceinline__ void load_row(const T* row, const Chunks& at, float (&x)[kN]) {
  float a[8], b[8];
  load(row + at.a, a);
  load(row + at.b, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = a[i];
    x[8 + i] = b[i];
  }
}
template <class T>
__device__ __forceinline__ void store_row(T* row, const Chunks& at, const float (&x)[kN]) {
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] = x[i];
    b[i] = x[8 + i];
  }
  store(row + at.a, a);
  store(row + at.b, b);
}

template <int LEVELS>
__device__ __forceinline__ float row_sum(float x) {
  return across<LEVELS>(x, [](float a, float b) { return a + b; });
}

// The angles of a lane's pairs; 1 and 0 outside the rotated part, NaN for a
// position that the tables do not hold (nothing is read for it).
__device__ __forceinline__ void angles(const Args& a, int lane, bool turned, int64_t b, int64_t t, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    c[j] = 1.0f;
    s[j] = 0.0f;
  }
  if (!turned) return;
  const int64_t pos = a.pos ? a.pos[b * a.ps[0] + t * a.ps[1]] : t;
  if (pos >= 0 && pos < a.table_rows) {
    load(a.cos + pos * (a.rot / 2) + 8 * lane, c);
    load(a.sin + pos * (a.rot / 2) + 8 * lane, s);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = s[j] = __builtin_nanf("");
  }
}

// LEVELS: a group has 2^LEVELS lanes.  HEADS: rows of a group.
// 32768 tokens of 20 heads of 128 in bf16: 62 us, 5.4 TB/s; in fp32 134 us, 5.0 TB/s; 64 tokens:
// 3.5 us, a launch and one row's chain of loads.
template <int DT, bool INTER, int LEVELS, int HEADS>
__global__ __launch_bounds__(kThreads) void qk_fwd_kernel(const Args a) {
  using T = typename Store<DT>::type;
  constexpr int kLanes = 1 << LEVELS;
  const bool keys = blockIdx.x >= a.first_k;
  const Side& side = a.s[keys];
  const uint32_t place = (blockIdx.x - (keys ? a.first_k : 0)) * (kThreads / kLanes) + threadIdx.x / kLanes;
  if (place >= side.units) return;
  const int unit = static_cast<int>(place), token = side.shares.divide(unit), first = (unit - token * static_cast<int>(side.shares.n)) * HEADS;
  const int lane = threadIdx.x % kLanes, b = a.tokens.divide(token), t = token - b * static_cast<int>(a.tokens.n);
  const Chunks at = chunks_of<INTER>(lane, a.d, a.rot);
  const T* x = static_cast<const T*>(side.x) + b * side.xs[0] + t * side.xs[1];
  Raw<T> raw[HEADS] = {};
#pragma unroll
  for (int j = 0; j < HEADS; ++j)
    if (at.some && first + j < side.heads) raw[j].load(x + (first + j) * side.xs[2], at);
  float w[kN] = {}, c[8], s[8];
  if (at.some) load_row(static_cast<const T*>(side.w), at, w);
  angles(a, lane, at.turned, b, t, c, s);
  T* y = static_cast<T*>(side.y) + (static_cast<int64_t>(token) * side.heads + first) * a.d;
#pragma unroll
  for (int j = 0; j < HEADS; ++j) {
    float u[kN], sum = 0.0f;
    raw[j].get(u);
#pragma unroll
    for (int i = 0; i < kN; ++i) sum += u[i] * u[i];
    const float r = 1.0f / sqrtf(row_sum<LEVELS>(sum) / a.d + a.eps);
#pragma unroll
    for (int i = 0; i < kN; ++i) u[i] = u[i] * r * w[i];
    if (at.turned) turn<INTER>(u, c, s);
    if (at.some && first + j < side.heads) store_row(y + j * a.d, at, u);
  }
}

// The sum over a wave's groups of 2^LEVELS lanes, lane by lane.  (The workgroup's groups
// added in pairs through LDS, both kinds in one workgroup: 9.1 us on 100 tokens of 24 heads,
// so 4.6.)
template <int LEVELS>
__device__ __forceinline__ float group_sum(float x) {
  if constexpr (LEVELS < 4) x += dpp<0x128 /* row_ror 8 */>(x);
  if constexpr (LEVELS < 3) x += dpp<0x124 /* row_ror 4 */>(x);
  const Two rows = halves16(x);
  const Two both = halves32(rows.a + rows.b);
  return both.a + both.b;
}

// 32768 tokens of 20 heads of 128 in bf16: 90 us with the second kernel's 5, 5.6 TB/s.
template <int DT, bool INTER, int LEVELS>
__global__ __launch_bounds__(kThreads) void qk_bwd_kernel(const Args a) {
  using T = typename Store<DT>::type;
  constexpr int kLanes = 1 << LEVELS, kGroups = kThreads / kLanes, kWaves = kThreads / kWave;
  __shared__ float sums[kWaves][kLanes * kN];
  const int lane = threadIdx.x % kLanes;
  const Chunks at = chunks_of<INTER>(lane, a.d, a.rot);
  const bool keys = blockIdx.x >= a.first_k;
  const Side& side = a.s[keys];
  const uint32_t first = blockIdx.x - (keys ? a.first_k : 0), groups = keys ? gridDim.x - a.first_k : a.first_k;
  float w[kN] = {}, dw[kN] = {};
  if (at.some) load_row(static_cast<const T*>(side.w), at, w);
  for (uint32_t place = first * kGroups + threadIdx.x / kLanes; place < side.units; place += groups * kGroups) {
    const int unit = static_cast<int>(place), token = side.shares.divide(unit), h = unit - token * static_cast<int>(side.shares.n);
    const int b = a.tokens.divide(token), t = token - b * static_cast<int>(a.tokens.n);
    Raw<T> rx = {}, rg = {};
    if (at.some) {
      rx.load(static_cast<const T*>(side.x) + b * side.xs[0] + t * side.xs[1] + h * side.xs[2], at);
      rg.load(static_cast<const T*>(side.dy) + b * side.ds[0] + t * side.ds[1] + h * side.ds[2], at);
    }
    float c[8], s[8];
    angles(a, lane, at.turned, b, t, c, s);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = -s[j];
    float u[kN], g[kN];
    rx.get(u);
    rg.get(g);
    if (at.turned) turn<INTER>(g, c, s);
    float sum = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      sum += u[i] * u[i];
      dot += g[i] * w[i] * u[i];
    }
    const float r = 1.0f / sqrtf(row_sum<LEVELS>(sum) / a.d + a.eps);
    const float mean = row_sum<LEVELS>(dot) * r / a.d;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float v = u[i] * r;
      dw[i] += g[i] * v;
      u[i] = r * (g[i] * w[i] - v * mean);
    }
    if (at.some) store_row(static_cast<T*>(side.y) + static_cast<int64_t>(unit) * a.d, at, u);
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const float sum = group_sum<LEVELS>(dw[i]);
    if (threadIdx.x % kWave < kLanes) sums[threadIdx.x / kWave][i * kLanes + lane] = sum;
  }
  __syncthreads();
  if (threadIdx.x >= kLanes * kN || !at.some) return;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) sum += sums[i][threadIdx.x];
  const int i = threadIdx.x / kLanes;
  a.parts[static_cast<int64_t>(blockIdx.x) * a.d + (i < 8 ? at.a + i : at.b + i - 8)] = sum;
}

// The sums of the workgroups' rows of d floats, those of the queries and then those of the
// keys: a workgroup takes 16 columns of one kind, 64 sums of every 64th row each, then adds
// those in pairs.
constexpr int kColumns = 16, kRows = 64;
__global__ __launch_bounds__(kColumns* kRows) void qk_sum_kernel(const float* parts, int rows_q, int rows_k, int d, float* dq_w, float* dk_w) {
  __shared__ float sums[kRows][kColumns];
  const int first = blockIdx.x * kColumns, row = threadIdx.x / kColumns;
  const bool keys = first >= d;
  const int col = first - (keys ? d : 0) + threadIdx.x % kColumns, end = keys ? rows_q + rows_k : rows_q;
  float sum = 0.0f;
#pragma unroll 8
  for (int r = (keys ? rows_q : 0) + row; r < end; r += kRows) sum += parts[static_cast<int64_t>(r) * d + col];
  sums[row][threadIdx.x % kColumns] = sum;
  for (int n = kRows / 2; n > 0; n /= 2) {
    __syncthreads();
    if (row < n) sums[row][threadIdx.x % kColumns] += sums[row + n][threadIdx.x % kColumns];
  }
  if (row == 0) {
    float* out = keys ? dk_w : dq_w;
    if (out) out[col] = sums[0][threadIdx.x];
  }
}

int check(const fewbit_qk* a) {
  if (!a) return FEWBIT_E_NULL;
  if (a->dtype < FEWBIT_F32 || a->dtype > FEWBIT_BF16) return FEWBIT_E_DTYPE;
  if (a->reserved != 0 || a->heads_q < 0 || a->heads_k < 0 || a->batch < 0 || a->tokens < 0 || a->table_rows < 0)
    return FEWBIT_E_INVALID;
  if (a->head_dim < 16 || a->head_dim > 256 || a->head_dim % 16 != 0) return FEWBIT_E_INVALID;
  if (a->rot < 0 || a->rot > a->head_dim || a->rot % 16 != 0) return FEWBIT_E_INVALID;
  if (a->interleaved != 0 && a->interleaved != 1) return FEWBIT_E_INVALID;
  if (!(a->eps >= 0.0f && std::isfinite(a->eps))) return FEWBIT_E_INVALID;
  if (a->heads_q > 1 << 16 || a->heads_k > 1 << 16) return FEWBIT_E_INVALID;
  if (a->tokens >= int64_t{1} << 31 || a->batch >= int64_t{1} << 31) return FEWBIT_E_INVALID;
  // rows are counted in 31 bits
  if (a->tokens > 0 && a->batch > 0 && (std::max(a->heads_q, a->heads_k) + 1) * a->tokens >= (int64_t{1} << 31) / a->batch)
    return FEWBIT_E_INVALID;
  return FEWBIT_OK;
}

bool nothing(const fewbit_qk* a) { return a->batch == 0 || a->tokens == 0 || a->heads_q + a->heads_k == 0; }

// Rows start at multiples of 16 bytes.
bool strides_fit(const fewbit_qk* a, const int64_t (&s)[3]) {
  const int64_t per = a->dtype == FEWBIT_F32 ? 4 : 8;
  return s[0] % per == 0 && s[1] % per == 0 && s[2] % per == 0;
}

int levels_of(int d) { return d <= 64 ? 2 : d <= 128 ? 3 : 4; }

// Rows of a group of the forward: two where that leaves eight waves per CU, else one.
// (32768 tokens of 20 heads in bf16: 63.7 us with two, 63.9 with four, 70.5 with one; 4096
// tokens of 24 heads of 64: 9.0, 8.9 and 8.4.)  The backward's groups take one row at a
// time, and several after one another (two at a time: 107 us to 97).
constexpr int kHeads = 2;
int heads_of(const fewbit_qk* a) {
  const int64_t groups = a->batch * a->tokens * ((a->heads_q + kHeads - 1) / kHeads + (a->heads_k + kHeads - 1) / kHeads);
  return groups >= static_cast<int64_t>(device_cus()) * 8 * (kWave >> levels_of(a->head_dim)) ? kHeads : 1;
}

// Workgroups for so many groups of lanes.
int64_t groups_of(const fewbit_qk* a, int64_t units) {
  const int64_t per = kThreads >> levels_of(a->head_dim);
  return (units + per - 1) / per;
}

Args args_of(const fewbit_qk* a, const float* cos, const float* sin, const int64_t* pos, bool back) {
  Args r{};
  for (int i = 0; i < 3; ++i) {
    r.s[0].xs[i] = a->q_stride[i];
    r.s[1].xs[i] = a->k_stride[i];
    r.s[0].ds[i] = a->dq_stride[i];
    r.s[1].ds[i] = a->dk_stride[i];
  }
  r.s[0].heads = a->heads_q;
  r.s[1].heads = a->heads_k;
  r.cos = cos;
  r.sin = sin;
  r.pos = pos;
  r.ps[0] = a->position_stride[0];
  r.ps[1] = a->position_stride[1];
  r.table_rows = a->table_rows;
  r.tokens = divisor(static_cast<int>(a->tokens));
  r.d = a->head_dim;
  r.rot = a->rot;
  r.eps = a->eps;
  const int heads = back ? 1 : heads_of(a);
  for (Side& side : r.s) {
    const int shares = (side.heads + heads - 1) / heads;
    side.shares = divisor(std::max(shares, 1));
    side.units = static_cast<uint32_t>(a->batch * a->tokens * shares);
  }
  r.first_k = static_cast<uint32_t>(groups_of(a, r.s[0].units));
  return r;
}

// Workgroups of the backward for the queries and for the keys: all take as many rows, and
// there are at most as many as the chip holds at once, five per CU, for each leaves a row
// for the second kernel.  (32768 tokens of 20 heads in bf16: 90 us; with four per CU 93, six
// 102, eight 95.)
struct Parts {
  int64_t q, k;
};
Parts parts_of(const fewbit_qk* a, const Args& r) {
  const int64_t q = groups_of(a, r.s[0].units), k = groups_of(a, r.s[1].units), most = 5 * static_cast<int64_t>(device_cus());
  const auto over = [](int64_t n, int64_t by) { return (n + by - 1) / by; };
  int64_t each = std::max<int64_t>(1, over(q + k, most));
  if (over(q, each) + over(k, each) > most) ++each;
  return {over(q, each), over(k, each)};
}

template <int DT, bool INTER, int LEVELS>
hipError_t start_at(const fewbit_qk* a, const Args& r, bool back, unsigned groups, hipStream_t s) {
  const bool several = heads_of(a) == kHeads;
  auto fwd = several ? qk_fwd_kernel<DT, INTER, LEVELS, kHeads> : qk_fwd_kernel<DT, INTER, LEVELS, 1>;
  return launch(back ? qk_bwd_kernel<DT, INTER, LEVELS> : fwd, dim3(groups), kThreads, s, r);
}
template <int DT, bool INTER>
hipError_t start_inter(const fewbit_qk* a, const Args& r, bool back, unsigned groups, hipStream_t s) {
  switch (levels_of(a->head_dim)) {
    case 2: return start_at<DT, INTER, 2>(a, r, back, groups, s);
    case 3: return start_at<DT, INTER, 3>(a, r, back, groups, s);
    default: return start_at<DT, INTER, 4>(a, r, back, groups, s);
  }
}
template <int DT>
hipError_t start_dt(const fewbit_qk* a, const Args& r, bool back, unsigned groups, hipStream_t s) {
  return a->interleaved ? start_inter<DT, true>(a, r, back, groups, s) : start_inter<DT, false>(a, r, back, groups, s);
}
hipError_t start(const fewbit_qk* a, const Args& r, bool back, unsigned groups, hipStream_t s) {
  return a->dtype == FEWBIT_F32   ? start_dt<FEWBIT_F32>(a, r, back, groups, s)
         : a->dtype == FEWBIT_F16 ? start_dt<FEWBIT_F16>(a, r, back, groups, s)
                                  : start_dt<FEWBIT_BF16>(a, r, back, groups, s);
}

// Checks that both directions make of what they read.
int check_inputs(const fewbit_qk* a, const void* q, const void* k, const void* qw, const void* kw, const float* cos,
                 const float* sin) {
  if (a->heads_q > 0 && (!q || !qw)) return FEWBIT_E_NULL;
  if (a->heads_k > 0 && (!k || !kw)) return FEWBIT_E_NULL;
  if (a->rot > 0 && a->table_rows > 0 && (!cos || !sin)) return FEWBIT_E_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(qw) || misaligned(kw) || misaligned(cos) || misaligned(sin))
    return FEWBIT_E_ALIGN;
  if ((a->heads_q > 0 && !strides_fit(a, a->q_stride)) || (a->heads_k > 0 && !strides_fit(a, a->k_stride)))
    return FEWBIT_E_ALIGN;
  return FEWBIT_OK;
}

}  // namespace

extern "C" int fewbit_qk_fwd(const fewbit_qk* a, const void* q, const void* k, const void* q_weight,
                             const void* k_weight, const float* cos, const float* sin, const int64_t* positions,
                             void* q_out, void* k_out, void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  if (nothing(a)) return FEWBIT_OK;
  rc = check_inputs(a, q, k, q_weight, k_weight, cos, sin);
  if (rc != FEWBIT_OK) return rc;
  if ((a->heads_q > 0 && !q_out) || (a->heads_k > 0 && !k_out)) return FEWBIT_E_NULL;
  if (misaligned(q_out) || misaligned(k_out)) return FEWBIT_E_ALIGN;
  Args r = args_of(a, cos, sin, positions, false);
  r.s[0].x = q;
  r.s[1].x = k;
  r.s[0].w = q_weight;
  r.s[1].w = k_weight;
  r.s[0].y = q_out;
  r.s[1].y = k_out;
  const int64_t groups = r.first_k + groups_of(a, r.s[1].units);
  if (!fits_launch(groups, kThreads)) return FEWBIT_E_INVALID;
  rc = check_stream_device(static_cast<hipStream_t>(stream));
  if (rc != FEWBIT_OK) return rc;
  return launch_status("fewbit_qk_fwd", start(a, r, false, static_cast<unsigned>(groups), static_cast<hipStream_t>(stream)));
}

extern "C" int64_t fewbit_qk_workspace(const fewbit_qk* a) {
  const int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  if (nothing(a)) return 0;
  const Parts parts = parts_of(a, args_of(a, nullptr, nullptr, nullptr, true));
  return (parts.q + parts.k) * a->head_dim * static_cast<int64_t>(sizeof(float));
}

extern "C" int fewbit_qk_bwd(const fewbit_qk* a, const void* dq_out, const void* dk_out, const void* q, const void* k,
                             const void* q_weight, const void* k_weight, const float* cos, const float* sin,
                             const int64_t* positions, void* dq, void* dk, float* dq_weight, float* dk_weight,
                             void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  const bool none = nothing(a);           // no rows: the weights' gradients are 0
  if ((a->heads_q > 0 && !dq_weight) || (a->heads_k > 0 && !dk_weight)) return FEWBIT_E_NULL;
  if (!none) {
    rc = check_inputs(a, q, k, q_weight, k_weight, cos, sin);
    if (rc != FEWBIT_OK) return rc;
    if ((a->heads_q > 0 && (!dq_out || !dq)) || (a->heads_k > 0 && (!dk_out || !dk)) || !workspace) return FEWBIT_E_NULL;
    if (misaligned(dq_out) || misaligned(dk_out) || misaligned(dq) || misaligned(dk) || misaligned(workspace))
      return FEWBIT_E_ALIGN;
    if ((a->heads_q > 0 && !strides_fit(a, a->dq_stride)) || (a->heads_k > 0 && !strides_fit(a, a->dk_stride)))
      return FEWBIT_E_ALIGN;
    if (workspace_bytes < fewbit_qk_workspace(a)) return FEWBIT_E_INVALID;
  }
  if (!dq_weight && !dk_weight) return FEWBIT_OK;         // no heads, and nothing to write zeros to
  rc = check_stream_device(static_cast<hipStream_t>(stream));
  if (rc != FEWBIT_OK) return rc;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Parts parts{0, 0};
  if (!none) {
    Args r = args_of(a, cos, sin, positions, true);
    r.s[0].x = q;
    r.s[1].x = k;
    r.s[0].w = q_weight;
    r.s[1].w = k_weight;
    r.s[0].dy = dq_out;
    r.s[1].dy = dk_out;
    r.s[0].y = dq;
    r.s[1].y = dk;
    r.parts = static_cast<float*>(workspace);
    parts = parts_of(a, r);
    r.first_k = static_cast<uint32_t>(parts.q);
    rc = launch_status("fewbit_qk_bwd", start(a, r, true, static_cast<unsigned>(parts.q + parts.k), s));
    if (rc != FEWBIT_OK) return rc;
  }
  return launch_status("fewbit_qk_bwd", launch(qk_sum_kernel, dim3(2 * a->head_dim / kColumns), kColumns * kRows, s,
                                               static_cast<const float*>(workspace), static_cast<int>(parts.q), static_cast<int>(parts.k),
                                               a->head_dim, dq_weight, dk_weight));
}
