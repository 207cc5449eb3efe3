// attention.hip -- attention and its gradient on the matrix cores.
//
// Definitions, layouts and masks are in fewbit_block.h.
//
// Rows.  The query heads that share a key head are rows of one problem: row r of
// a (sequence, key head) is head r % G of query r / G, G query heads to a key
// head.  So keys and values are read once for all of them, and the gradients of
// shared keys and values add up in registers, in a fixed order.
//
// Orientation.  A 32x32 product of the matrix cores leaves column n in lanes n
// and n + 32, rows 8 (i / 4) + 4 (lane / 32) + i % 4 in registers i = 0..15.  The
// scores are formed so that the axis summed over next lies in registers: S^T = K
// Q^T (a lane is a row of Q) in the forward and for dQ, S = Q K^T (a lane is a
// key) for dK and dV.  Then softmax statistics are one number per lane, and P
// goes into the next product as its second operand without leaving the
// registers: that operand holds, in lane n, eight values k = 8 (lane / 32) + j,
// and any order of k does when both operands have the same.  The first operand
// of the second product is V^T (or K^T, dO^T, Q^T): read from the row-major tile
// in LDS by the transposing load, four rows at a time, in that order.
//
// Tiles lie in LDS row-major in 16-byte chunks, chunk c of row r at c ^ f(r) (swizzle).
//
// Times of long walks differ by 5% from card to card, with the clock that the matrix cores
// hold: ranges are those of several.
#include <algorithm>
#include <type_traits>

#include "block.h"

namespace {

using namespace block;

constexpr float kLog2e = 1.44269504088896340736f;

template <int DT>
struct Mma;
template <>
struct Mma<FEWBIT_BF16> {
  using T = __bf16;
  typedef __bf16 V8 __attribute__((ext_vector_type(8)));
  typedef __bf16 V4 __attribute__((ext_vector_type(4)));
  typedef float C __attribute__((ext_vector_type(16)));
  static __device__ __forceinline__ C mul(V8 a, V8 b, C c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma<FEWBIT_F16> {
  using T = _Float16;
  typedef _Float16 V8 __attribute__((ext_vector_type(8)));
  typedef _Float16 V4 __attribute__((ext_vector_type(4)));
  typedef float C __attribute__((ext_vector_type(16)));
  static __device__ __forceinline__ C mul(V8 a, V8 b, C c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Args {
  const void *q, *k, *v, *dout, *out;
  void *o, *dq, *dk, *dv;
  float* lse;
  float* stats;                       // backward: lse * log2(e) of every row (infinity if it is empty), then delta; lifted
  int64_t stats_delta;
  float *part_o, *part_lse;           // forward: results that are to be joined
  float *part_dq, *part_dkv;          // backward: the same
  const int32_t *cu_q, *cu_k, *k_len;
  int64_t qs[3], ks[3], vs[3], ds[3];
  int64_t rows_q, rows_k;
  int batch, hq, hkv, g, d;           // g: query heads to a key head
  int causal, window;
  float scale;
  Divisor by_g, by_hkv, by_place, by_parts, by_parts_dkv, by_quads, by_rows;
  int tiles, tiles_first;             // of a sequence; whether all sequences' first tiles come first
  int rows;                           // split forward: of a sequence and key head
  int shares, share_least;            // split forward: workgroups of a key head, passes of one at least
  int parts, parts_dkv;               // of a workgroup's walk (forward or dQ; dK and dV)
};

// One (sequence, key head): where its rows begin and how many there are.
struct Seq {
  int64_t q0, k0;       // first row in the tensors (packed) or 0
  int64_t b;            // sequence for the strides and dense layouts (packed: 0)
  int nq, nk;
};

__device__ __forceinline__ int clamped(int x, int64_t most) { return static_cast<int>(min(static_cast<int64_t>(max(x, 0)), most)); }

// Rows of 64 packed sequences from b0 on in one of the tensors, one to a lane, of whose offsets
// in cu (the last entry's past the end) the lane has its own and the next; sequence `batch` are
// the rows past the last.  An offset below one before it counts as that one, so no row is in
// two sequences.  `past`: where the sequence before b0 ended, and then where the last of these
// did.
struct Span {
  int at, end;
};
__device__ __forceinline__ Span offsets_of(const int32_t* cu, int batch, int b) { return {cu[min(b, batch)], cu[min(b + 1, batch)]}; }
__device__ __forceinline__ Span spans(Span s, int64_t rows, int batch, int b0, int& past) {
  const int lane = threadIdx.x % kWave, b = b0 + lane, all = static_cast<int>(rows);
  s.at = b == 0 ? 0 : b > batch ? all : max(clamped(s.at, rows), past);
  s.end = b >= batch ? all : max(clamped(s.end, rows), past);
  if (__any(s.end < s.at)) {
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
      const int other = __shfl_up(s.at, step);
      if (lane >= step) s.at = max(s.at, other);
    }
    s.end = max(s.at, s.end);
  }
  past = __builtin_amdgcn_readlane(s.end, kWave - 1);
  return s;
}

// The sequence and tile that place `at` of the tiles of all sequences stands for,
// `rows` rows (times `times`) to a tile; false past the last.  Rows of no sequence
// come last; they see, and are seen by, nothing.  Offsets of 256 sequences are on their way
// together, and only where the place is found are tiles counted lane by lane: 65536 rows of 12
// heads of 64 in 1024 sequences, forward, 207 us; counted for each 64 one after another 337.
__device__ __forceinline__ bool find_packed(const Args& a, bool keys, int times, int rows, int at, Seq& s, int& tile, int& tiles) {
  constexpr int kTurns = 4;
  const int lane = threadIdx.x % kWave;
  const bool alike = a.cu_q == a.cu_k && a.rows_q == a.rows_k;
  int before = 0, past_q = 0, past_k = 0;
  for (int first = 0; first <= a.batch; first += kTurns * kWave) {
    Span qs[kTurns], ks[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      qs[t] = offsets_of(a.cu_q, a.batch, first + t * kWave + lane);
      if (!alike) ks[t] = offsets_of(a.cu_k, a.batch, first + t * kWave + lane);
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int b0 = first + t * kWave;
      if (b0 > a.batch) break;
      const Span q = spans(qs[t], a.rows_q, a.batch, b0, past_q), k = alike ? q : spans(ks[t], a.rows_k, a.batch, b0, past_k);
      const int nq = q.end - q.at, nk = k.end - k.at;
      const int own = static_cast<int>((static_cast<int64_t>(keys ? nk : nq) * times + rows - 1) / rows);
      const int all = wave_sum(own);
      if (at >= before + all) {
        before += all;
        continue;
      }
      int sum = own;                                          // of this lane's and all before it
#pragma unroll
      for (int step = 1; step < kWave; step *= 2) {
        const int other = __shfl_up(sum, step);
        if (lane >= step) sum += other;
      }
      const int l = __builtin_ctzll(__ballot(at < before + sum));
      tiles = __builtin_amdgcn_readlane(own, l);
      tile = at - before - __builtin_amdgcn_readlane(sum - own, l);
      s.b = 0;
      s.q0 = __builtin_amdgcn_readlane(q.at, l);
      s.k0 = __builtin_amdgcn_readlane(k.at, l);
      s.nq = __builtin_amdgcn_readlane(nq, l);
      s.nk = __builtin_amdgcn_readlane(nk, l);
      if (b0 + l == a.batch) (keys ? s.nq : s.nk) = 0;
      return true;
    }
  }
  return false;
}

// This workgroup's key head, sequence and tile.  Neighbouring workgroups have
// different key heads, so those of one key head, which read the same keys, run on
// one XCD where the heads are a multiple of eight.  Tiles come from the last, which under a
// causal mask see the most keys, to the first: those of one sequence after another, so that
// its keys are read from that XCD's L2, or (tiles_first) the last ones of all sequences first.
__device__ __forceinline__ bool find(const Args& a, bool keys, int times, int rows, int place, Seq& s, int& tile) {
  if (a.cu_q) {
    int tiles;
    if (!find_packed(a, keys, times, rows, place, s, tile, tiles)) return false;
    tile = keys ? tile : tiles - 1 - tile;
    return true;
  }
  const int by = a.by_place.divide(place), rest = place - by * static_cast<int>(a.by_place.n);
  s.b = a.tiles_first ? rest : by;
  tile = a.tiles_first ? by : rest;
  if (!keys) tile = a.tiles - 1 - tile;       // of keys the first are seen by the most rows
  s.q0 = s.k0 = 0;
  s.nq = static_cast<int>(a.rows_q);
  s.nk = a.k_len ? clamped(a.k_len[s.b], a.rows_k) : static_cast<int>(a.rows_k);
  return true;
}

// The first and one past the last key that query `pos` sees.
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range keys_of(const Args& a, const Seq& s, int pos) {
  const int here = pos + s.nk - s.nq;           // below 2^30 either way, as the window is
  Range r{0, s.nk};
  if (a.causal) r.hi = min(max(here + 1, 0), s.nk);
  if (a.window) r.lo = min(max(here + 1 - a.window, 0), s.nk);
  return r;
}

// Keys that any of a workgroup's rows sees, and rows of all sequences and heads.
constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kRowsWave = 32, kRowsGroup = kWaves * kRowsWave;      // rows of a wave and of a workgroup
__device__ __forceinline__ Range keys_of_group(const Args& a, const Seq& s, int first, int rows) {
  return {keys_of(a, s, a.by_g.divide(first)).lo, keys_of(a, s, a.by_g.divide(min(first + kRowsGroup, rows) - 1)).hi};
}
__device__ __forceinline__ int64_t rows_all(const Args& a) { return (a.cu_q ? 1 : a.batch) * a.rows_q * a.hq; }

// Rows (query * G + head) that see key j, and that see any of a workgroup's keys; keys
// of all sequences and heads.
__device__ __forceinline__ Range rows_of_key(int g, int causal, int window, const Seq& s, int j) {
  const int here = j - s.nk + s.nq;             // the query that stands at key j
  Range r{0, s.nq * g};
  if (causal) r.lo = min(max(here, 0), s.nq) * g;
  if (window) r.hi = min(max(here + window, 0), s.nq) * g;
  if (j >= s.nk) r.hi = 0;
  return r;
}
__device__ __forceinline__ Range rows_of_keys(const Args& a, const Seq& s, int first, int n) {
  if (first >= s.nk) return {0, 0};
  return {rows_of_key(a.g, a.causal, a.window, s, first).lo, rows_of_key(a.g, a.causal, a.window, s, min(first + n, s.nk) - 1).hi};
}
__device__ __forceinline__ int64_t keys_all(const Args& a) { return (a.cu_q ? 1 : a.batch) * a.rows_k * a.hkv; }

// Sixteen lanes that read a chunk each of rows one after another, and 32 lanes of a
// transposing read, which take 64 bytes of four rows, then touch every bank once.
template <int D>
__device__ __forceinline__ int swizzle(int row) {
  return D == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
}

// Elements that rows may lie apart for a lane's offset inside a load to fit 31 bits.
constexpr int64_t kNear = int64_t{1} << 26;

template <class T>
__device__ __forceinline__ const T* uniform(const T* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x >> 32));
  return reinterpret_cast<const T*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Brings a tile of ROWS rows of D elements to LDS, 16 bytes a lane and load, without
// registers between.  A load writes 1 KiB of LDS in lane order, so the swizzle is in
// which chunk of its row a lane asks for.  Rows past the last are read as the last,
// chunks past head_dim as the first: what multiplies them is 0 (masked scores; the
// other operand's elements past head_dim) or is not stored.
// POLICY: cache policy of the loads, kNt for what is read once.
template <int DT, int D, int ROWS, int WAVES, int POLICY = 0>
struct Stage {
  using T = typename Mma<DT>::T;
  static constexpr int kChunks = D / 8, kRowsLoad = kWave / kChunks, kLoads = ROWS / kRowsLoad / WAVES;
  static constexpr int kKinds = 16 / (kRowsLoad * WAVES) > 1 ? 16 / (kRowsLoad * WAVES) : 1;      // of swizzles among a wave's loads
  static_assert(ROWS % (kRowsLoad * WAVES) == 0, "whole loads for every wave");
  int wave, row, chunk[kKinds];

  __device__ __forceinline__ Stage(int d, int wave_) : wave(__builtin_amdgcn_readfirstlane(wave_)) {
    const int lane = threadIdx.x % kWave;
    row = lane / kChunks;
#pragma unroll
    for (int j = 0; j < kKinds; ++j) {
      const int c = (lane % kChunks) ^ swizzle<D>(row + row_of(j));
      chunk[j] = c * 8 < d ? c * 8 : 0;
    }
  }
  __device__ __forceinline__ int row_of(int j) const { return (j * WAVES + wave) * kRowsLoad; }
  // at(i): where row i of the tile begins
  template <class F>
  __device__ __forceinline__ void issue(T* lds, F at) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load(at(row + row_of(j)) + chunk[j % kKinds], lds, j);
  }
  // The same for rows `stride` apart from `base` on (the same for all lanes), at most
  // kNear: the address is a scalar and a lane's offset, its row's and its chunk's.
  __device__ __forceinline__ void issue(T* lds, const T* base, int64_t stride, uint32_t apart) const {
    asm volatile("" : "+v"(apart));             // the sums are not kept in registers
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(uniform(base + row_of(j) * stride)) + (apart + chunk[j % kKinds] * 2)), lds, j);
  }
  // The same with an offset of its own for every load.
  __device__ __forceinline__ void issue(T* lds, const T* base, const uint32_t (&offset)[kLoads]) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(uniform(base)) + offset[j]), lds, j);
  }
  template <class F>
  __device__ __forceinline__ void offsets(F at, uint32_t (&offset)[kLoads]) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) offset[j] = static_cast<uint32_t>(at(row + row_of(j)) + chunk[j % kKinds]) * 2;
  }

 private:
  __device__ __forceinline__ void load(const T* p, T* lds, int j) const {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)(lds + row_of(j) * D), 16, 0, POLICY);
  }
};

// Rows first .. of a tensor as a walk over tiles of ROWS wants them: whole tiles of
// rows not too far apart by the quick way, the others with each row's own address.
template <int DT, int D, int ROWS, int WAVES, int POLICY = 0>
struct Rows {
  using T = typename Mma<DT>::T;
  using S = Stage<DT, D, ROWS, WAVES, POLICY>;
  const T* base;
  int64_t stride;
  int last;             // the last row there is
  bool near;
  uint32_t apart;       // bytes between the first row and this lane's of a load
  __device__ __forceinline__ Rows(const S& stage, const T* base_, int64_t stride_, int last_)
      : base(base_), stride(stride_), last(last_), near(stride_ < kNear), apart(static_cast<uint32_t>(stage.row * static_cast<int>(stride_)) * 2) {}
  __device__ __forceinline__ void issue(const S& stage, T* lds, int first) const {
    if (near && first + ROWS - 1 <= last)
      stage.issue(lds, base + first * stride, stride, apart);
    else
      stage.issue(lds, [&](int i) { return base + min(first + i, last) * stride; });
  }
};

// Where there are few workgroups, several share one's walk: part `part` of `parts` of
// the passes of `step` that it takes to get through `all`, two passes at least each; how
// many parts there are then.
constexpr int kPassesPart = 2;
struct Slice {
  Range r;
  int used;
};
__device__ __forceinline__ Slice slice_of(Range all, int step, int parts, int part) {
  const int begin = all.lo / step * step, n = all.hi > begin ? (all.hi - begin + step - 1) / step : 0;
  if (parts == 1) return {{begin, all.hi}, 1};
  const int per = max(kPassesPart, (n + parts - 1) / parts);
  return {{begin + part * per * step, min(all.hi, begin + (part + 1) * per * step)}, max(1, (n + per - 1) / per)};
}

// A workgroup's key head, part of the walk and place.
struct Spot {
  int hk, part, place;
};
__device__ __forceinline__ Spot spot_of(const Divisor& by_hkv, const Divisor& by_parts) {
  const int id = static_cast<int>(blockIdx.x), rest = by_hkv.divide(id), place = by_parts.divide(rest);
  return {id - rest * static_cast<int>(by_hkv.n), rest - place * static_cast<int>(by_parts.n), place};
}

// Two tiles that come and are worked on together.
template <class T, int N>
struct Pair {
  __attribute__((aligned(16))) T a[N];
  __attribute__((aligned(16))) T b[N];
};

// All but the last N of this wave's loads to LDS are done.
template <int N>
__device__ __forceinline__ void landed() {
  static_assert(N < 16, "one field of the wait's operand");
  __builtin_amdgcn_s_waitcnt(0x0f70 | N);       // vmcnt(N), nothing else
}

// Walks tiles at, at + step, .. < end through two buffers: while one is worked on the
// next tile comes into the other.  (Buffers are apart so that the compiler does not make
// reads of one wait for loads into the other.)
template <class Buffer, class Issue, class Work>
__device__ __forceinline__ void walk(int at, int step, int end, Buffer& a, Buffer& b, Issue issue, Work work) {
  if (at >= end) return;
  issue(a, at);
  for (; at < end; at += 2 * step) {
    landed<0>();
    __syncthreads();
    if (at + step < end) issue(b, at + step);
    work(a, at);
    if (at + step >= end) break;
    landed<0>();
    __syncthreads();
    if (at + 2 * step < end) issue(a, at + 2 * step);
    work(b, at + step);
  }
}

// First operand from rows: lane m holds row `row0 + m % 32`, elements 16 step + 8
// (lane / 32) ..+7.
template <int DT, int D>
struct RowReader {
  using T = typename Mma<DT>::T;
  using V8 = typename Mma<DT>::V8;
  int at;       // in bytes
  // A copy whose addresses are formed where they are used: the compiler else keeps the
  // address of every read of a tile in a register of its own throughout.
  __device__ __forceinline__ RowReader here() const {
    RowReader r = *this;
    asm volatile("" : "+v"(r.at));
    return r;
  }
  __device__ __forceinline__ RowReader() {
    const int lane = threadIdx.x % kWave, row = lane % 32;
    at = (row * D + ((lane / 32) ^ swizzle<D>(row)) * 8) * 2;
  }
  __device__ __forceinline__ V8 read(const T* lds, int row0, int step) const {
    return *reinterpret_cast<const V8*>(reinterpret_cast<const char*>(lds + row0 * D) + (at ^ (step * 32)));
  }
};

// First operand from columns: lane m holds column 32 tile + m % 32, of the rows
// row0 + 8 (j / 4) + 4 (lane / 32) + j % 4, j = 0..7.  Of 16 lanes that read
// together, lane i points at four elements of row i / 4 and receives element i of
// each row.
template <int DT, int D>
struct ColumnReader {
  using T = typename Mma<DT>::T;
  using V8 = typename Mma<DT>::V8;
  int at;
  __device__ __forceinline__ ColumnReader here() const {
    ColumnReader r = *this;
    asm volatile("" : "+v"(r.at));
    return r;
  }
  __device__ __forceinline__ ColumnReader() {
    const int lane = threadIdx.x % kWave, i = lane % 16, row = 4 * (lane / 32) + i / 4;
    const int chunk = 2 * (lane / 16 % 2) + i % 4 / 2;
    at = (row * D + (chunk ^ swizzle<D>(row)) * 8 + i % 2 * 4) * 2;
  }
  __device__ __forceinline__ s16x4 four(const T* lds, int row0, int tile, int up) const {
    // row0 is a multiple of 16; rows 8 further on have another bit of the swizzle
    const char* p = reinterpret_cast<const char*>(lds + (row0 + 8 * up) * D) + (at ^ (tile * 64) ^ (up * 32));
    using L = __attribute__((address_space(3))) s16x4*;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((L)const_cast<char*>(p));
  }
  __device__ __forceinline__ V8 read(const T* lds, int row0, int tile) const {
    const s16x4 a = four(lds, row0, tile, 0), b = four(lds, row0, tile, 1);
    return __builtin_bit_cast(V8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Second operand from registers 8 step ..+7 of a product.
template <int DT>
__device__ __forceinline__ typename Mma<DT>::V8 narrow(const f32x16& x, int step) {
  typename Mma<DT>::V8 r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = static_cast<typename Mma<DT>::T>(x[8 * step + j]);
  return r;
}

// A row of a tensor as second operand: elements 16 step + 8 (lane / 32) ..+7 of the
// lane's row, zeros past head_dim (and, with ZERO, for a row that is not there).
template <int DT, int D, bool ZERO = false>
__device__ __forceinline__ void load_rows(const typename Mma<DT>::T* row, int d, typename Mma<DT>::V8 (&x)[D / 16], bool there = true) {
  using V8 = typename Mma<DT>::V8;
  const int c = threadIdx.x % kWave / 32 * 8;
  if (d == D) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) x[s] = *reinterpret_cast<const V8*>(row + 16 * s + c);
  } else {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      x[s] = V8{};
      if (16 * s + c < d) x[s] = *reinterpret_cast<const V8*>(row + 16 * s + c);
    }
  }
  if (ZERO && !there) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) x[s] = V8{};
  }
}

// Registers of D / 32 products whose lane is a row of the result, 32 elements each, times
// `scale`, to `offset` elements past `base`, the lane's row's; the first `rows` rows are there.
// They go through 32 D elements of LDS of the wave's own, so that a store has whole rows, 16
// bytes a lane: a lane's own elements lie in fours with another lane's between.  16 x 2048
// rows, 16 heads of 128, on 64 keys: 71 us, stored from the registers 87; 16 x 2048 causal rows,
// forward 373 us to 381, dK and dV 831 to 838, dQ 510 to 503.
template <int DT, int D>
__device__ __forceinline__ void store_rows(typename Mma<DT>::T* lds, int d, const f32x16 (&x)[D / 32], float scale, typename Mma<DT>::T* base,
                                           uint32_t offset, int rows) {
  using T = typename Mma<DT>::T;
  using V4 = typename Mma<DT>::V4;
  using V8 = typename Mma<DT>::V8;
  constexpr int kChunks = D / 8, kRowsStore = kWave / kChunks;
  // of 16 rows' chunks, no two in the same banks
  const auto place = [](int row, int chunk) { return row * D + (chunk ^ (D == 128 ? row & 15 : row >> 1 & 7)) * 8; };
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      V4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = static_cast<T>(x[t][4 * u + j] * scale);
      *reinterpret_cast<V4*>(lds + place(lane % 32, 4 * t + u) + lane / 32 * 4) = y;
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int chunk = lane % kChunks;
#pragma unroll
  for (int i = 0; i < 32 / kRowsStore; ++i) {
    const int r = i * kRowsStore + lane / kChunks;
    const uint32_t row = __shfl(offset, r);
    const V8 y = *reinterpret_cast<const V8*>(lds + place(r, chunk));
    if (r < rows && chunk * 8 < d) *reinterpret_cast<V8*>(base + row + chunk * 8) = y;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The lane's row as fp32, from the registers.
template <int D>
__device__ __forceinline__ void store_rows32(float* row, int d, const f32x16 (&x)[D / 32], float scale) {
  const int c = threadIdx.x % kWave / 32 * 4;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = 32 * t + 8 * u + c;
      if (at < d) *reinterpret_cast<f32x4*>(row + at) = f32x4{x[t][4 * u], x[t][4 * u + 1], x[t][4 * u + 2], x[t][4 * u + 3]} * scale;
    }
}

__device__ __forceinline__ int key_of(int i) { return 8 * (i / 4) + i % 4; }      // plus 4 (lane / 32)

// ---------------------------------------------------------------- forward
// Softmax statistics and output of the lane's row.  `most` is what exponentials are
// taken from: a score of the row, at most kSlack (of base-2 logarithms) under its largest
// so far.  Sums and outputs are rescaled only where a score exceeds that, not for every
// new maximum; nothing is lost by it, exponentials below 2^kSlack round as those below 1.
constexpr float kSlack = 8.0f;
template <int D>
struct Running {
  float most = -INFINITY, sum = 0.0f;       // sum: of this lane's half of the keys
  f32x16 o[D / 32] = {};
};

// The probabilities (from x.most) of SUBS runs of 32 keys from key k0 of the sequence
// on, their keys in lk.
template <int DT, int D, int SUBS>
__device__ __forceinline__ void score(const typename Mma<DT>::T* lk, int k0, const typename Mma<DT>::V8 (&q)[D / 16],
                                      const RowReader<DT, D>& rows, bool masked, Range r, float scale2, Running<D>& x,
                                      f32x16 (&s)[SUBS]) {
  const int half = threadIdx.x % kWave / 32 * 4;
#pragma unroll
  for (int u = 0; u < SUBS; ++u) {
    s[u] = f32x16{};
#pragma unroll
    for (int step = 0; step < D / 16; ++step) s[u] = Mma<DT>::mul(rows.read(lk, 32 * u, step), q[step], s[u]);
  }
  if (masked) {
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + 32 * u + key_of(i) + half;
        if (key < r.lo || key >= r.hi) s[u][i] = -INFINITY;
      }
  }
  float most = x.most;
#pragma unroll
  for (int u = 0; u < SUBS; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, s[u][i]);
  const Two both = halves32(most);
  most = fmaxf(both.a, both.b);
  if (__any((most - x.most) * scale2 > kSlack)) {
    const float base = most == -INFINITY ? 0.0f : most * scale2;
    const float fade = __builtin_amdgcn_exp2f(x.most * scale2 - base);
    x.sum *= fade;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) x.o[t][i] *= fade;
    x.most = most;
  }
  const float base = x.most == -INFINITY ? 0.0f : x.most * scale2;
  float sum = 0.0f;
#pragma unroll
  for (int u = 0; u < SUBS; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[u][i] = __builtin_amdgcn_exp2f(s[u][i] * scale2 - base);
      sum += s[u][i];
    }
  x.sum += sum;
}

// Adds up the values, in lv, by their probabilities.
template <int DT, int D, int SUBS>
__device__ __forceinline__ void gather(const typename Mma<DT>::T* lv, const ColumnReader<DT, D>& columns,
                                       const f32x16 (&s)[SUBS], Running<D>& x) {
#pragma unroll
  for (int u = 0; u < SUBS; ++u)
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      const auto p = narrow<DT>(s[u], step);
#pragma unroll
      for (int t = 0; t < D / 32; ++t) x.o[t] = Mma<DT>::mul(columns.read(lv, 32 * u + 16 * step, t), p, x.o[t]);
    }
}

constexpr int kKeys = 64;                                           // keys of a pass

// store_rows for rows of a (sequence, key head) from row `first` of all `rows` on; the lane's
// is head `head` of query `pos`.
template <int DT, int D>
__device__ __forceinline__ void store_queries(const Args& a, const Seq& s, void* out, typename Mma<DT>::T* lds, int hk, int first, int rows, int pos,
                                              int head, const f32x16 (&x)[D / 32], float scale) {
  const int pos0 = a.by_g.divide(first), head0 = hk * a.g;
  // below 2^32: 32 queries of at most 2^20 heads
  const uint32_t offset = (static_cast<uint32_t>(pos - pos0) * a.hq + (head - head0)) * a.d;
  store_rows<DT, D>(lds, a.d, x, scale, static_cast<typename Mma<DT>::T*>(out) + ((s.b * a.rows_q + s.q0 + pos0) * a.hq + head0) * a.d, offset,
                    rows - first);
}

// The forward for many rows: a workgroup holds 128 rows of Q in registers, 32 to a wave,
// and walks the keys they see in tiles of 64, one pass with a running maximum and sum; a
// tile of K and V (32 KB at D = 128) serves all four waves, and two workgroups share a CU.
// The maximum follows only when a row's scores pass it by 2^8, so the sums seldom have to
// be scaled.  Bound by the products and the exponentials between them, which two waves a
// SIMD overlap in part: 4 x 4096 rows, 16 heads of 128 in bf16, 554 to 579 us, 950 to 990
// TFLOP/s (a library product of 8192^3 reaches 1160), matrix pipes busy for 53% of the cycles;
// 16 x 2048, causal, 358 to 376 us, 45%.  Of a workgroup's time 10 us pass outside the tiles.
// Forming the next tile's scores beside this tile's exponentials was slower, 625 us to 560.
template <int DT, int D>
__global__ __launch_bounds__(kThreads, 2) void attn_fwd_kernel(const Args a) {
  using T = typename Mma<DT>::T;
  __shared__ Pair<T, kKeys * D> buf0, buf1;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const auto [hk, part, place] = spot_of(a.by_hkv, a.by_parts);
  Seq s;
  int tile;
  if (!find(a, false, a.g, kRowsGroup, place, s, tile)) return;
  const int rows = s.nq * a.g, first = tile * kRowsGroup;
  if (first >= rows) return;
  const int row = first + wave * kRowsWave + lane % 32;
  const bool there = row < rows;
  const int pos = a.by_g.divide(min(row, rows - 1)), head = hk * a.g + min(row, rows - 1) - pos * a.g;
  typename Mma<DT>::V8 q[D / 16];
  load_rows<DT, D>(static_cast<const T*>(a.q) + s.b * a.qs[0] + (s.q0 + pos) * a.qs[1] + head * a.qs[2], a.d, q);

  // keys that any row of the workgroup sees, that this lane's row sees, and that
  // all rows of the wave see
  const Slice slice = slice_of(keys_of_group(a, s, first, rows), kKeys, a.parts, part);
  const Range all = slice.r;
  if (part >= slice.used) return;
  const Range own = keys_of(a, s, pos);
  const int w0 = min(first + wave * kRowsWave, rows - 1), w1 = min(first + wave * kRowsWave + kRowsWave, rows) - 1;
  const int p0 = a.by_g.divide(w0), p1 = a.by_g.divide(max(w1, w0));
  const Range every{keys_of(a, s, p1).lo, keys_of(a, s, p0).hi};

  const T* kb = static_cast<const T*>(a.k) + s.b * a.ks[0] + s.k0 * a.ks[1] + hk * a.ks[2];
  const T* vb = static_cast<const T*>(a.v) + s.b * a.vs[0] + s.k0 * a.vs[1] + hk * a.vs[2];
  const Stage<DT, D, kKeys, kWaves> stage(a.d, wave);
  const Rows<DT, D, kKeys, kWaves> keys(stage, kb, a.ks[1], s.nk - 1), values(stage, vb, a.vs[1], s.nk - 1);
  const RowReader<DT, D> rr;
  const ColumnReader<DT, D> cr;
  Running<D> x;
  walk(all.lo, kKeys, all.hi, buf0, buf1,
       [&](Pair<T, kKeys * D>& to, int k0) {
         keys.issue(stage, to.a, k0);
         values.issue(stage, to.b, k0);
       },
       [&](const Pair<T, kKeys * D>& in, int k0) {
         f32x16 p[kKeys / 32];
         score<DT, D, kKeys / 32>(in.a, k0, q, rr, k0 < every.lo || k0 + kKeys > every.hi, own, a.scale * kLog2e, x, p);
         gather<DT, D, kKeys / 32>(in.b, cr, p, x);
       });
  const Two both = halves32(x.sum);
  const float sum = both.a + both.b;
  const float lse = sum == 0.0f ? -INFINITY : x.most * a.scale + logf(sum);
  const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  const int64_t at = (s.b * a.rows_q + s.q0 + pos) * a.hq + head;
  if (slice.used == 1) {
    __syncthreads();                    // the tiles' buffers are free
    const int w = __builtin_amdgcn_readfirstlane(wave);
    store_queries<DT, D>(a, s, a.o, reinterpret_cast<T*>(&buf0) + w * 32 * D, hk, first + w * kRowsWave, rows, pos, head, x.o, inverse);
    if (there && lane < 32) a.lse[(s.b * a.hq + head) * a.rows_q + s.q0 + pos] = lse;
  } else if (there) {
    const int64_t to = part * rows_all(a) + at;
    store_rows32<D>(a.part_o + to * a.d, a.d, x.o, inverse);
    if (lane < 32) a.part_lse[to] = lse;
  }
}

// Few rows over many keys (single tokens over a cache): a unit is a sequence and key head
// of at most 32 rows, and its keys are taken in passes of 128.  The passes of all
// sequences, in one line, are cut into equal shares, one to a workgroup: whatever the
// lengths of the caches, all workgroups end at the same time.  A workgroup's waves take
// different keys of each pass and add their results up at the end of the unit, or of the
// share; what belongs to a unit that is not all in one share is left in the workspace and
// added by a second kernel.  Share w and unit u meet at most once, and of all meetings in
// line each has the next w or the next u: w + u numbers them.
constexpr int kKeysSplit = 32 * kWaves;

// Unit `unit`: its sequence, and the keys that its rows see, from a multiple of 32 on.
struct Unit {
  Seq s;
  int rows;
  Range keys;
  int passes;           // at least one
};
__device__ __forceinline__ Unit unit_of(const Args& a, int unit) {
  Unit u;
  u.s.b = unit;
  u.s.q0 = u.s.k0 = 0;
  u.s.nq = static_cast<int>(a.rows_q);
  u.s.nk = a.k_len ? clamped(a.k_len[unit], a.rows_k) : static_cast<int>(a.rows_k);
  u.rows = u.s.nq * a.g;
  u.keys.lo = keys_of(a, u.s, 0).lo / 32 * 32;
  u.keys.hi = max(u.keys.lo, keys_of(a, u.s, u.s.nq - 1).hi);
  u.passes = max(1, (u.keys.hi - u.keys.lo + kKeysSplit - 1) / kKeysSplit);
  return u;
}

// All units' passes in line: passes of a share, and of all units, and those before unit
// `stop`.  Units are alike where no sequence is shorter.
struct Line {
  int share, all, before;
};
__device__ __forceinline__ Line line_of(const Args& a, int stop) {
  Line l;
  if (!a.k_len) {
    const int each = unit_of(a, 0).passes;
    l.all = each * a.batch;
    l.before = each * stop;
  } else {
    const int lane = threadIdx.x % kWave, units = a.batch;
    int all = 0, before = 0;
    for (int u = lane; u < units; u += kWave) {
      const int n = unit_of(a, u).passes;
      all += n;
      if (u < stop) before += n;
    }
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
      all += __shfl_xor(all, step);
      before += __shfl_xor(before, step);
    }
    l.all = __builtin_amdgcn_readfirstlane(all);
    l.before = __builtin_amdgcn_readfirstlane(before);
  }
  l.share = max(a.share_least, (l.all + a.shares - 1) / a.shares);
  return l;
}

// The unit that pass `at` of the line is in, and which of its passes it is.
__device__ __forceinline__ int unit_at(const Args& a, int at, int& pass) {
  if (!a.k_len) {
    const int each = unit_of(a, 0).passes, unit = at / each;
    pass = at - unit * each;
    return unit;
  }
  const int lane = threadIdx.x % kWave, units = a.batch;
  int before = 0;
  for (int u0 = 0; u0 < units; u0 += kWave) {
    const int own = u0 + lane < units ? unit_of(a, u0 + lane).passes : 0;
    int sum = own;
#pragma unroll
    for (int step = 1; step < kWave; step *= 2) {
      const int other = __shfl_up(sum, step);
      if (lane >= step) sum += other;
    }
    const uint64_t past = __ballot(at < before + sum);
    if (past) {
      const int first = __builtin_ctzll(past);
      pass = __builtin_amdgcn_readfirstlane(at - before - __shfl(sum - own, first));
      return __builtin_amdgcn_readfirstlane(u0 + first);
    }
    before += __builtin_amdgcn_readfirstlane(__shfl(sum, kWave - 1));
  }
  pass = 0;
  return units;
}

// Bound by HBM: one row on 64 caches of up to 8192 keys, 270000 in all, 16 heads to 4 of 128
// in bf16, 553 MB, 100 us, 5.5 TB/s.  Each wave has two buffers of its own, so that it waits for
// no other.  Keys are read once and not kept in the caches (64 caches of 8192 keys each, more
// than the memory-side cache holds: 177 us, else 200).
template <int DT, int D>
__global__ __launch_bounds__(kThreads, 2) void attn_split_kernel(const Args a) {
  using T = typename Mma<DT>::T;
  __shared__ __attribute__((aligned(16))) T lk[kWaves][32 * D], lv[kWaves][32 * D];
  __shared__ float stats[kWaves][2][32];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int share = a.by_hkv.divide(blockIdx.x), hk = static_cast<int>(blockIdx.x) - share * a.hkv;
  const Line line = line_of(a, 0);
  if (share > (line.all - 1) / line.share) return;
  int at = share * line.share;
  const int end = at + min(line.share, line.all - at);
  int pass;
  for (int unit = unit_at(a, at, pass); at < end; ++unit, pass = 0) {
    const Unit u = unit_of(a, unit);
    const Seq& s = u.s;
    const int passes = min(u.passes - pass, end - at);
    const bool whole = passes == u.passes;
    at += passes;
    // This lane's query and head; asked for again behind the loop, which has no registers
    // to keep them in.
    struct Mine {
      int pos, head;
      bool there;
    };
    const auto mine = [&]() __attribute__((always_inline)) {
      int l = lane;
      asm volatile("" : "+v"(l));
      const int row = l % 32, some = min(row, u.rows - 1), pos = a.by_g.divide(some);
      return Mine{pos, hk * a.g + some - pos * a.g, row < u.rows};
    };
    const auto [pos, head, there] = mine();
    const Range own = keys_of(a, s, pos);
    const Range every{keys_of(a, s, s.nq - 1).lo, keys_of(a, s, 0).hi};
    Range all;
    all.lo = u.keys.lo + pass * kKeysSplit;
    all.hi = min(u.keys.hi, all.lo + passes * kKeysSplit);
    Running<D> x;
    if (all.lo < all.hi) {
      typename Mma<DT>::V8 q[D / 16];
      load_rows<DT, D>(static_cast<const T*>(a.q) + s.b * a.qs[0] + pos * a.qs[1] + head * a.qs[2], a.d, q);
      const T* kb = static_cast<const T*>(a.k) + s.b * a.ks[0] + hk * a.ks[2];
      const T* vb = static_cast<const T*>(a.v) + s.b * a.vs[0] + hk * a.vs[2];
      const Stage<DT, D, 32, 1, kNt> stage(a.d, 0);
      const Rows<DT, D, 32, 1, kNt> keys(stage, kb, a.ks[1], all.hi - 1), values(stage, vb, a.vs[1], all.hi - 1);
      const RowReader<DT, D> rr;
      const ColumnReader<DT, D> cr;
      // Each wave has buffers of its own: while it works on keys the next keys, and while
      // it works on values the next values, are on their way.
      constexpr int kLoads = decltype(stage)::kLoads;
      int k0 = all.lo + 32 * wave;
      if (k0 < all.hi) {
        keys.issue(stage, lk[wave], k0);
        values.issue(stage, lv[wave], k0);
      }
      for (; k0 < all.hi; k0 += kKeysSplit) {
        f32x16 p[1];
        landed<kLoads>();
        score<DT, D, 1>(lk[wave], k0, q, rr.here(), k0 < every.lo || k0 + 32 > min(every.hi, all.hi), Range{own.lo, min(own.hi, all.hi)},
                        a.scale * kLog2e, x, p);
        keys.issue(stage, lk[wave], k0 + kKeysSplit);       // past the end: the last row, again and again
        landed<kLoads>();
        gather<DT, D, 1>(lv[wave], cr.here(), p, x);
        values.issue(stage, lv[wave], k0 + kKeysSplit);
      }
      landed<0>();
    }
    const auto [pos2, head2, there2] = mine();
    // The waves' results.  Wave t adds up all waves' columns 32 t ..+31 and writes them;
    // the others' come through LDS, three parts for each t.
    const Two both = halves32(x.sum);
    if (lane < 32) {
      stats[wave][0][lane] = x.most;
      stats[wave][1][lane] = both.a + both.b;
    }
    __syncthreads();
    float most = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, stats[w][0][lane % 32]);
    const float base = most == -INFINITY ? 0.0f : most, scale2 = a.scale * kLog2e;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      sum += stats[w][1][lane % 32] * __builtin_amdgcn_exp2f((stats[w][0][lane % 32] - base) * scale2);
    const float fade = __builtin_amdgcn_exp2f((x.most - base) * scale2);
    const auto parts = [&](int t) { return reinterpret_cast<float*>(t < D / 64 ? lk : lv) + t % (D / 64) * 3 * 16 * kWave + lane; };
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      if (wave == t) continue;
      float* to = parts(t) + (wave - (wave > t)) * 16 * kWave;
#pragma unroll
      for (int i = 0; i < 16; ++i) to[i * kWave] = x.o[t][i] * fade;
    }
    __syncthreads();
    const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const float lse = sum == 0.0f ? -INFINITY : most * a.scale + logf(sum);
    const int64_t part = (static_cast<int64_t>(share + unit) * a.hkv + hk) * a.rows + lane % 32;
    if (there2 && wave == 0 && lane < 32) (whole ? a.lse[(s.b * a.hq + head2) * a.rows_q + pos2] : a.part_lse[part]) = lse;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      if (wave != t) continue;
      const float* from = parts(t);
      float o[16];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        o[i] = (x.o[t][i] * fade + from[i * kWave] + from[(16 + i) * kWave] + from[(32 + i) * kWave]) * inverse;
#pragma unroll
      for (int c4 = 0; c4 < 4; ++c4) {
        const int c = 32 * t + 8 * c4 + lane / 32 * 4;
        if (!there2 || c >= a.d) continue;
        const f32x4 y{o[4 * c4], o[4 * c4 + 1], o[4 * c4 + 2], o[4 * c4 + 3]};
        if (whole)
          *reinterpret_cast<typename Mma<DT>::V4*>(static_cast<T*>(a.o) + ((s.b * a.rows_q + pos2) * a.hq + head2) * a.d + c) =
              __builtin_convertvector(y, typename Mma<DT>::V4);
        else
          *reinterpret_cast<f32x4*>(a.part_o + part * a.d + c) = y;
      }
    }
    __syncthreads();
  }
}

// Rows of units that several shares worked on: out = sum of their outputs, each by its
// weight exp(lse_share - lse).  A workgroup takes a row, each wave every fourth share, four
// at a time so that their loads are on their way together, two elements a lane.  Bound by
// latency: 4 to 6 us (one row on 16000 keys in 63 shares: 17 us with the shares' kernel, with
// one wave to a row 32).
constexpr int kSharesTurn = 4;
template <int DT>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(const Args a) {
  using T = typename Mma<DT>::T;
  __shared__ float2 sums[kWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int rest = a.by_rows.divide(blockIdx.x), of = static_cast<int>(blockIdx.x) - rest * a.rows;
  const int unit = a.by_hkv.divide(rest), hk = rest - unit * a.hkv;
  const Unit u = unit_of(a, unit);
  if (of >= u.rows) return;
  const Line line = line_of(a, unit);
  const int first = line.before / line.share, n = (line.before + u.passes - 1) / line.share - first + 1;
  if (n == 1) return;
  const int64_t step = static_cast<int64_t>(a.hkv) * a.rows;
  const int64_t part = (static_cast<int64_t>(first + unit) * a.hkv + hk) * a.rows + of;
  float most = -INFINITY;
  for (int i = lane; i < n; i += kWave) most = fmaxf(most, a.part_lse[part + i * step]);
  most = across<6>(most, [](float x, float y) { return fmaxf(x, y); });
  const float base = most == -INFINITY ? 0.0f : most;
  const float* o = a.part_o + part * a.d + (2 * lane < a.d ? 2 * lane : 0);
  float sum = 0.0f;
  float2 x{0.0f, 0.0f};
  for (int i0 = 0; i0 < n; i0 += kWave) {
    const float weight = i0 + lane < n ? __builtin_amdgcn_exp2f((a.part_lse[part + (i0 + lane) * step] - base) * kLog2e) : 0.0f;
    sum += weight;
    for (int i1 = wave; i1 < min(n - i0, kWave); i1 += kWaves * kSharesTurn) {
      float2 y[kSharesTurn];
#pragma unroll
      for (int k = 0; k < kSharesTurn; ++k) y[k] = *reinterpret_cast<const float2*>(o + min(i0 + i1 + k * kWaves, n - 1) * step * a.d);
#pragma unroll
      for (int k = 0; k < kSharesTurn; ++k) {
        const int i = i1 + k * kWaves;
        if (i0 + i >= n || i >= kWave) break;
        const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), i));
        x.x += w * y[k].x;
        x.y += w * y[k].y;
      }
    }
  }
  sum = across<6>(sum, [](float x, float y) { return x + y; });
  sums[wave][lane] = x;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    x.x += sums[w][lane].x;
    x.y += sums[w][lane].y;
  }
  const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  const int pos = a.by_g.divide(of), head = hk * a.g + of - pos * a.g;
  if (2 * lane < a.d) {
    T* out = static_cast<T*>(a.o) + ((u.s.b * a.rows_q + pos) * a.hq + head) * a.d + 2 * lane;
    out[0] = static_cast<T>(x.x * inverse);
    out[1] = static_cast<T>(x.y * inverse);
  }
  if (lane == 0) a.lse[(u.s.b * a.hq + head) * a.rows_q + pos] = sum == 0.0f ? -INFINITY : base + logf(sum);
}

// The same for the parts of a workgroup's walk over keys: a thread takes four elements of
// a row, with the loads of four parts on their way together.  Bound by latency, 6 us.
constexpr int kPartsMost = 16, kPartsTurn = 4;
template <int DT>
__global__ __launch_bounds__(kThreads) void attn_parts_kernel(const Args a, Divisor by_joins) {
  using T = typename Mma<DT>::T;
  const auto [hk, join, place] = spot_of(a.by_hkv, by_joins);
  Seq s;
  int tile;
  if (!find(a, false, a.g, kRowsGroup, place, s, tile)) return;
  const int rows = s.nq * a.g, first = tile * kRowsGroup, i = join * kThreads + static_cast<int>(threadIdx.x);
  const int of = a.by_quads.divide(i), c = (i - of * static_cast<int>(a.by_quads.n)) * 4, row = first + of;
  if (of >= kRowsGroup || row >= rows) return;
  const int used = slice_of(keys_of_group(a, s, first, rows), kKeys, a.parts, 0).used;
  if (used == 1) return;
  const int pos = a.by_g.divide(row), head = hk * a.g + row - pos * a.g;
  const int64_t at = (s.b * a.rows_q + s.q0 + pos) * a.hq + head, step = rows_all(a);
  float lse[kPartsMost], most = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int k = 0; k < kPartsMost; ++k) lse[k] = k < used ? a.part_lse[k * step + at] : -INFINITY;
#pragma unroll
  for (int k = 0; k < kPartsMost; ++k) most = fmaxf(most, lse[k]);
  const float base = most == -INFINITY ? 0.0f : most;
  f32x4 o{};
#pragma unroll
  for (int k0 = 0; k0 < kPartsMost; k0 += kPartsTurn) {
    if (k0 >= used) break;
    f32x4 parts[kPartsTurn];
#pragma unroll
    for (int k = 0; k < kPartsTurn; ++k) parts[k] = *reinterpret_cast<const f32x4*>(a.part_o + (min(k0 + k, used - 1) * step + at) * a.d + c);
#pragma unroll
    for (int k = 0; k < kPartsTurn; ++k) {
      const float w = __builtin_amdgcn_exp2f((lse[k0 + k] - base) * kLog2e);
      sum += w;
      if (k0 + k < used) o += parts[k] * w;
    }
  }
  const float inverse = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  *reinterpret_cast<typename Mma<DT>::V4*>(static_cast<T*>(a.o) + at * a.d + c) = __builtin_convertvector(o * inverse, typename Mma<DT>::V4);
  if (c == 0) a.lse[(s.b * a.hq + head) * a.rows_q + s.q0 + pos] = sum == 0.0f ? -INFINITY : base + logf(sum);
}

// ---------------------------------------------------------------- backward
// The kernel for dK and dV forms 2^15 P, which it hands over in fp16 whatever the storage
// type: 11 bits, for small probabilities too (bf16's eight would be rounded a second time
// in dS: dK's error 0.0030 of its norm instead of 0.0025).
constexpr int kLift = 15;

// dS in fp16.  Gradients without a loss scale are small, and dS is smaller by P: below 2^-14
// fp16 has fewer bits the smaller a number is.  So dS goes into its products as 2^lift dS, lift
// being a lane's own, of a row for dQ and of a key for dK: it begins where no number that fp16
// inputs give is lost, and where one passes fp16's largest it falls until that has the exponent
// kHalfAim, and the sums so far with it.  2048 rows and keys, 2 heads of 64, dO of 1e-4: dQ and
// dK are off by 0.0047 of their norm, as the exact gradients are when rounded; with dS itself
// 0.027.  The backward of 16 x 2048 rows, 16 heads of 64, takes 1145 us so and 1075 without; of
// 4 x 4096, 16 heads of 128, 1922 and 1902.
constexpr int kHalfLift = 60, kHalfAim = 10;
constexpr float kHalfMost = 65504.0f;
template <int D>
__device__ __forceinline__ void fit_half(f32x16& ds, f32x16 (&sums)[D / 32], int& lift) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(ds[i]));
  if (!__any(most > kHalfMost)) return;
  const Two both = halves32(most);            // both lanes of a column
  most = fmaxf(both.a, both.b);
  const int down = most > kHalfMost ? static_cast<int>(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - kHalfAim : 0;
  const float by = ldexpf(1.0f, -down);
#pragma unroll
  for (int i = 0; i < 16; ++i) ds[i] *= by;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[t][i] *= by;
  lift -= down;
}

// With P from lse, delta_i = <dO_i, O_i>, dP = dO V^T and dS = P (dP - delta):
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
// dQ needs all keys of a row and dK, dV all rows of a key: one kernel for each,
// both of which form S and dP (seven products where five would do, but no sums
// across workgroups: nothing is added atomically, and no gradient waits in memory).
//
// dQ: 128 rows of Q and dO to a workgroup, which walks tiles of 64 keys as the forward does;
// delta is formed from their rows and left for the other kernel.  dS is rounded to the storage
// type for its product with K.  Bound as the forward is: 4 x 4096 rows, 16 heads of 128 in
// bf16, 742 to 791 us, 1040 to 1110 TFLOP/s, matrix pipes busy for 58%; 16 x 2048, causal, 488
// to 516 us, 46%.
constexpr int kFewKeys = 16, kThinWindow = 4;
template <int DT, int D>
__global__ __launch_bounds__(kThreads, 2) void attn_dq_kernel(const Args a) {
  using T = typename Mma<DT>::T;
  using V8 = typename Mma<DT>::V8;
  __shared__ Pair<T, kKeys * D> buf0, buf1;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const auto [hk, part, place] = spot_of(a.by_hkv, a.by_parts);
  Seq s;
  int tile;
  if (!find(a, false, a.g, kRowsGroup, place, s, tile)) return;
  const int rows = s.nq * a.g, first = tile * kRowsGroup;
  if (first >= rows) return;
  const Slice slice = slice_of(keys_of_group(a, s, first, rows), kKeys, a.parts, part);
  const Range all = slice.r;
  if (part >= slice.used) return;
  const int row = first + wave * kRowsWave + lane % 32;
  const bool there = row < rows;
  const int pos = a.by_g.divide(min(row, rows - 1)), head = hk * a.g + min(row, rows - 1) - pos * a.g;
  const int64_t at = ((s.b * a.rows_q + s.q0 + pos) * a.hq + head) * a.d;
  const int64_t stat = (s.b * a.hq + head) * a.rows_q + s.q0 + pos;
  V8 q[D / 16], dout[D / 16];
  load_rows<DT, D>(static_cast<const T*>(a.q) + s.b * a.qs[0] + (s.q0 + pos) * a.qs[1] + head * a.qs[2], a.d, q);
  load_rows<DT, D>(static_cast<const T*>(a.dout) + s.b * a.ds[0] + (s.q0 + pos) * a.ds[1] + head * a.ds[2], a.d, dout);
  float delta = 0.0f;
  {
    V8 o[D / 16];
    load_rows<DT, D>(static_cast<const T*>(a.out) + at, a.d, o);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) delta += static_cast<float>(o[i][j]) * static_cast<float>(dout[i][j]);
    const Two both = halves32(delta);
    delta = both.a + both.b;
  }
  float lse = there ? a.lse[stat] : -INFINITY;
  lse = lse == -INFINITY ? INFINITY : lse * kLog2e;           // of an empty row no key is seen

  const Range own = keys_of(a, s, pos);
  const int w0 = min(first + wave * kRowsWave, rows - 1), w1 = min(first + wave * kRowsWave + kRowsWave, rows) - 1;
  const int p0 = a.by_g.divide(w0), p1 = a.by_g.divide(max(w1, w0));
  const Range every{keys_of(a, s, p1).lo, keys_of(a, s, p0).hi};
  const Range any{keys_of(a, s, p0).lo, keys_of(a, s, p1).hi};

  const T* kb = static_cast<const T*>(a.k) + s.b * a.ks[0] + s.k0 * a.ks[1] + hk * a.ks[2];
  const T* vb = static_cast<const T*>(a.v) + s.b * a.vs[0] + s.k0 * a.vs[1] + hk * a.vs[2];
  const Stage<DT, D, kKeys, kWaves> stage(a.d, wave);
  const Rows<DT, D, kKeys, kWaves> keys(stage, kb, a.ks[1], s.nk - 1), values(stage, vb, a.vs[1], s.nk - 1);
  const RowReader<DT, D> rows_at;
  const ColumnReader<DT, D> columns_at;
  const float scale2 = a.scale * kLog2e;
  const auto issue = [&](Pair<T, kKeys * D>& to, int k0) {
    keys.issue(stage, to.a, k0);
    values.issue(stage, to.b, k0);
  };
  // S (-infinity where the mask hides it) and dP of 32 keys of a tile
  const auto products = [&](const Pair<T, kKeys * D>& in, const RowReader<DT, D>& rr, int k0, int u, bool masked, f32x16& p,
                            f32x16& dp) __attribute__((always_inline)) {
    p = dp = f32x16{};
#pragma unroll
    for (int step = 0; step < D / 16; ++step) {
      p = Mma<DT>::mul(rr.read(in.a, 32 * u, step), q[step], p);
      dp = Mma<DT>::mul(rr.read(in.b, 32 * u, step), dout[step], dp);
    }
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + 32 * u + key_of(i) + lane / 32 * 4;
        if (key < own.lo || key >= own.hi) p[i] = -INFINITY;
      }
    }
  };
  const auto hidden = [&](int k0) { return k0 < every.lo || k0 + kKeys > every.hi; };      // from some row of the wave
  f32x16 dq[D / 32] = {};
  int lift = DT == FEWBIT_F16 ? kHalfLift : 0;
  // dS (times 2^lift) of 32 keys into dQ
  const auto add = [&](const Pair<T, kKeys * D>& in, const ColumnReader<DT, D>& cr, int u, f32x16& ds) __attribute__((always_inline)) {
    if constexpr (DT == FEWBIT_F16) fit_half<D>(ds, dq, lift);
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      const V8 n = narrow<DT>(ds, step);
#pragma unroll
      for (int t = 0; t < D / 32; ++t) dq[t] = Mma<DT>::mul(cr.read(in.a, 32 * u + 16 * step, t), n, dq[t]);
    }
  };
  // Rows that see few keys: the rounding of out is in delta, and the larger beside their dS the fewer
  // they are.  Where a workgroup's first row sees at most kFewKeys, delta is sum_j P_ij dP_ij for all
  // rows that see no key past the first tile, whose P and dP stay in registers meanwhile; with a
  // window of at most kThinWindow, for all rows, formed ahead.  (16 causal rows in bf16: dQ is 0.0030
  // of its norm off with delta from out, 0.0023 so, its rounding alone 0.0017.  Only the thin windows
  // take longer for it: 4 x 4096 rows, 16 heads of 128, forward apart, 251 us, else 226.)
  const Range seen = keys_of_group(a, s, first, rows), least = keys_of(a, s, a.by_g.divide(first));
  const int begin = seen.lo / kKeys * kKeys;
  int next = all.lo;
  if (least.hi - least.lo <= kFewKeys && next == begin && next < all.hi) {
    if (a.window > 0 && a.window <= kThinWindow) {
      float sum = 0.0f;
      walk(begin, kKeys, seen.hi, buf0, buf1, issue, [&](const Pair<T, kKeys * D>& in, int k0) {
        if (k0 + kKeys <= any.lo || k0 >= any.hi) return;
        const auto rr = rows_at.here();
        const bool masked = hidden(k0);
#pragma unroll
        for (int u = 0; u < kKeys / 32; ++u) {
          f32x16 p, dp;
          products(in, rr, k0, u, masked, p, dp);
#pragma unroll
          for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(p[i] * scale2 - lse) * dp[i];
        }
      });
      const Two both = halves32(sum);
      delta = both.a + both.b;
    } else {
      next += kKeys;
      issue(buf0, begin);
      landed<0>();
      __syncthreads();
      if (any.lo < next && any.hi > begin) {
        f32x16 p[kKeys / 32], dp[kKeys / 32];
        const auto rr = rows_at.here();
        const auto cr = columns_at.here();
        const bool masked = hidden(begin);
        float sum = 0.0f;
#pragma unroll
        for (int u = 0; u < kKeys / 32; ++u) {
          products(buf0, rr, begin, u, masked, p[u], dp[u]);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            p[u][i] = __builtin_amdgcn_exp2f(p[u][i] * scale2 - lse);
            sum += p[u][i] * dp[u][i];
          }
        }
        const Two both = halves32(sum);
        if (own.hi <= next) delta = both.a + both.b;
#pragma unroll
        for (int u = 0; u < kKeys / 32; ++u) {
          const float up = DT == FEWBIT_F16 ? ldexpf(1.0f, lift) : 1.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) p[u][i] *= (dp[u][i] - delta) * up;
          add(buf0, cr, u, p[u]);
        }
      }
    }
    __syncthreads();                    // the tiles' buffers are free
  }
  walk(next, kKeys, all.hi, buf0, buf1, issue, [&](const Pair<T, kKeys * D>& in, int k0) {
    if (k0 + kKeys <= any.lo || k0 >= any.hi) return;
    const auto rr = rows_at.here();
    const auto cr = columns_at.here();
    const bool masked = hidden(k0);
#pragma unroll
    for (int u = 0; u < kKeys / 32; ++u) {
      const float from = lse - lift;
      f32x16 p, dp;
      products(in, rr, k0, u, masked, p, dp);
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(p[i] * scale2 - from) * (dp[i] - delta);
      add(in, cr, u, p);
    }
  });
  if (there && lane < 32 && part == 0) {
    a.stats[stat] = lse - kLift;
    a.stats[a.stats_delta + stat] = ldexpf(delta, -kLift);
  }
  const float scale = ldexpf(a.scale, -lift);
  if (slice.used == 1) {
    __syncthreads();                    // the tiles' buffers are free
    store_queries<DT, D>(a, s, a.dq, reinterpret_cast<T*>(&buf0) + wave * 32 * D, hk, first + wave * kRowsWave, rows, pos, head, dq, scale);
  } else if (there) {
    store_rows32<D>(a.part_dq + part * rows_all(a) * a.d + at, a.d, dq, scale);
  }
}

// A workgroup takes 4 runs of 32 SUBS keys and walks the rows that see them, 32 at a
// time.  Two waves share a run: one forms S, P and dV, the other dP, dS and dK, one
// tile of rows behind, with P handed over in LDS.  So each wave holds one of K and V
// and one of the two gradients, the same products run on both sides, and the two waves
// of a SIMD are always one of either kind.  The tiles come through three buffers.  P and
// dS are rounded to the storage type for their products with dO and Q.
// Bound by the products, the hand-over between them and 13 us of a workgroup's time outside
// the tiles, one workgroup to a CU: 4 x 4096 rows, 16 heads of 128 in bf16, 1210 to 1300 us,
// 850 to 910 TFLOP/s, matrix pipes busy for 45% of the cycles; 16 x 2048, causal, 784 to 823 us,
// 37%.  4 x 4096 rows, when these pairs took 1590 us: one wave for both sides, with twice the
// registers, 2430; 64 keys to a pair, which spills at D = 128, 1700.
constexpr int kRowsPass = 64;
constexpr int kPairs = 4, kThreadsPairs = 2 * kPairs * kWave;

template <int DT, int D, int SUBS>
__global__ __launch_bounds__(kThreadsPairs, 2) void attn_dkv_kernel(const Args a) {
  using T = typename Mma<DT>::T;
  using V8 = typename Mma<DT>::V8;
  constexpr int kRun = 32 * SUBS, kGroup = kPairs * kRun;
  struct Buffer : Pair<T, kRowsPass * D> {        // rows of Q and dO
    __attribute__((aligned(16))) float stats[2][kRowsPass];
  };
  __shared__ Buffer buf0, buf1, buf2;
  using Handed = typename Mma<FEWBIT_F16>::V8;
  __shared__ Handed handed[2][kPairs][SUBS][kRowsPass / 16][kWave];
  const int lane = threadIdx.x % kWave;
  const auto [hk, part, place] = spot_of(a.by_hkv, a.by_parts_dkv);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), pair = wave % kPairs;
  const bool second = wave >= kPairs;             // of a pair: dP, dS and dK
  Seq s;
  int tile;
  if (!find(a, true, 1, kGroup, place, s, tile)) return;
  // keys past those that are there have gradients too: zeros
  const int keys = a.cu_k ? s.nk : static_cast<int>(a.rows_k), first = tile * kGroup;
  if (first >= keys) return;
  const int run = first + pair * kRun;
  const Slice slice = slice_of(rows_of_keys(a, s, first, kGroup), kRowsPass, a.parts_dkv, part);
  const Range all = slice.r;
  if (part >= slice.used) return;
  V8 kv[SUBS][D / 16];
  {
    const T* base = second ? static_cast<const T*>(a.v) + s.b * a.vs[0] + s.k0 * a.vs[1] + hk * a.vs[2]
                           : static_cast<const T*>(a.k) + s.b * a.ks[0] + s.k0 * a.ks[1] + hk * a.ks[2];
    const int64_t stride = second ? a.vs[1] : a.ks[1];
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      const int key = run + 32 * u + lane % 32;
      load_rows<DT, D, true>(base + min(key, max(s.nk - 1, 0)) * stride, a.d, kv[u], key < s.nk);
    }
  }

  const int rows = s.nq * a.g;
  const auto rows_of = [g = a.g, causal = a.causal, window = a.window, s](int j) __attribute__((always_inline)) { return rows_of_key(g, causal, window, s, j); };
  const Range every{rows_of(run + kRun - 1).lo, run + kRun <= s.nk ? rows_of(run).hi : 0};      // that all keys of the run are seen by
  const Range any{rows_of(run).lo, run < s.nk ? rows_of(min(run + kRun, s.nk) - 1).hi : 0};      // that any is

  const T* qb = static_cast<const T*>(a.q) + s.b * a.qs[0] + s.q0 * a.qs[1] + static_cast<int64_t>(hk) * a.g * a.qs[2];
  const T* db = static_cast<const T*>(a.dout) + s.b * a.ds[0] + s.q0 * a.ds[1] + static_cast<int64_t>(hk) * a.g * a.ds[2];
  const int64_t sb = (s.b * a.hq + static_cast<int64_t>(hk) * a.g) * a.rows_q + s.q0;
  const Stage<DT, D, kRowsPass, kPairs> stage(a.d, pair);
  const T* base = second ? db : qb;
  const int64_t pos_stride = second ? a.ds[1] : a.qs[1], head_stride = second ? a.ds[2] : a.qs[2];
  // with a power of two of heads to a key head, rows of whole tiles lie alike in all tiles
  const int g_bits = __builtin_ctz(a.g);
  const bool near = a.g == 1 << g_bits && a.g <= kRowsPass && pos_stride < kNear / 16 && head_stride < kNear / 16;
  uint32_t offset[decltype(stage)::kLoads];
  stage.offsets([&](int i) { return (i >> g_bits) * static_cast<int>(pos_stride) + (i & (a.g - 1)) * static_cast<int>(head_stride); }, offset);
  const auto issue = [&](Buffer& to, int r0) __attribute__((always_inline)) {
    // the first waves of the pairs bring Q and lse, the second dO and delta
    T* lds = second ? to.b : to.a;
    if (near && r0 + kRowsPass <= rows)
      stage.issue(lds, base + static_cast<int64_t>(r0 >> g_bits) * pos_stride, offset);
    else
      stage.issue(lds, [&](int i) {
        const int r = min(r0 + i, rows - 1), pos = a.by_g.divide(r);
        return base + pos * pos_stride + (r - pos * a.g) * head_stride;
      });
    if (pair == 0) {                 // lse for the first, delta for the second
      const int r = min(r0 + lane, rows - 1), pos = a.by_g.divide(r);
      const float* p = a.stats + (second ? a.stats_delta : 0) + sb + (r - pos * a.g) * a.rows_q + pos;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                       (__attribute__((address_space(3))) void*)to.stats[second], 4, 0, 0);
    }
  };
  const RowReader<DT, D> rows_at;
  const ColumnReader<DT, D> columns_at;
  f32x16 acc[SUBS][D / 32] = {};
  int lift[SUBS];
#pragma unroll
  for (int u = 0; u < SUBS; ++u) lift[u] = DT == FEWBIT_F16 ? kHalfLift : 0;
  constexpr float lower = 1.0f / (1 << kLift);
  const float scale2 = a.scale * kLog2e;
  // One side's part of a tile of rows: SECOND and MASKED are constants, so that each
  // is one run of code in which products and the rest overlap.
  const auto work = [&](auto SECOND, auto MASKED, const Buffer& in, int r0, int slot) __attribute__((always_inline)) {
    const T *x = SECOND ? in.b : in.a, *y = SECOND ? in.a : in.b;
    const auto rr = rows_at.here();
    const auto cr = columns_at.here();
#pragma unroll
    for (int h = 0; h < kRowsPass / 32; ++h) {
      f32x16 p[SUBS] = {};
#pragma unroll
      for (int step = 0; step < D / 16; ++step) {
        const V8 row = rr.read(x, 32 * h, step);
#pragma unroll
        for (int u = 0; u < SUBS; ++u) p[u] = Mma<DT>::mul(row, kv[u][step], p[u]);
      }
      V8 n[SUBS][2];
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        if (MASKED) {
          const Range own = rows_of(run + 32 * u + lane % 32);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = r0 + 32 * h + key_of(i) + lane / 32 * 4;
            if (r < own.lo || r >= own.hi) p[u][i] = -INFINITY;
          }
        }
        const float up = SECOND && DT == FEWBIT_F16 ? ldexpf(1.0f, lift[u]) : 1.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x4 stat = *reinterpret_cast<const f32x4*>(&in.stats[SECOND][32 * h + 8 * c + lane / 32 * 4]);
          const Handed given = SECOND ? handed[slot][pair][u][2 * h + c / 2][lane] : Handed{};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = 4 * c + j;
            p[u][i] = SECOND ? static_cast<float>(given[i % 8]) * (p[u][i] * lower - stat[j])
                             : __builtin_amdgcn_exp2f(p[u][i] * scale2 - stat[j]);
            if (SECOND && DT == FEWBIT_F16) p[u][i] *= up;
          }
        }
        if constexpr (SECOND && DT == FEWBIT_F16) fit_half<D>(p[u], acc[u], lift[u]);
#pragma unroll
        for (int step = 0; step < 2; ++step) {
          n[u][step] = narrow<DT>(p[u], step);
          if (!SECOND) handed[slot][pair][u][2 * h + step][lane] = narrow<FEWBIT_F16>(p[u], step);
        }
      }
#pragma unroll
      for (int step = 0; step < 2; ++step)
#pragma unroll
        for (int t = 0; t < D / 32; ++t) {
          const V8 column = cr.read(y, 32 * h + 16 * step, t);
#pragma unroll
          for (int u = 0; u < SUBS; ++u) acc[u][t] = Mma<DT>::mul(column, n[u][step], acc[u][t]);
        }
    }
  };

  // turn i: tile i + 1 comes, the pairs' first waves work on tile i and their second
  // waves on tile i - 1
  const int begin = all.lo, tiles = all.hi > begin ? (all.hi - begin + kRowsPass - 1) / kRowsPass : 0;
  const auto turn = [&](Buffer& now, Buffer& before, Buffer& next, int i) __attribute__((always_inline)) {
    landed<0>();
    __syncthreads();
    if (i + 1 < tiles) issue(next, begin + (i + 1) * kRowsPass);
    const int r0 = begin + i * kRowsPass;
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    const int mine = second ? r0 - kRowsPass : r0;            // rows that none of the run's keys is seen by are left out
    if (mine + kRowsPass <= any.lo || mine >= any.hi) return;
    if (second) {
      if (i > 0) work(yes, no, before, mine, (i - 1) & 1);
    } else if (i < tiles) {
      if (r0 < every.lo || r0 + kRowsPass > every.hi)
        work(no, yes, now, r0, i & 1);
      else
        work(no, no, now, r0, i & 1);
    }
  };
  if (tiles > 0) {
    issue(buf0, begin);
    for (int i = 0; i <= tiles; i += 3) {
      turn(buf0, buf2, buf1, i);
      if (i + 1 > tiles) break;
      turn(buf1, buf0, buf2, i + 1);
      if (i + 2 > tiles) break;
      turn(buf2, buf1, buf0, i + 2);
    }
  }
  __syncthreads();                      // the tiles' buffers are free
  T* own = reinterpret_cast<T*>(second ? &buf1 : &buf0) + pair * 32 * D;
#pragma unroll
  for (int u = 0; u < SUBS; ++u) {
    const int key = run + 32 * u;
    const int64_t at = (s.b * a.rows_k + s.k0 + key) * a.hkv + hk;
    const float scale = second ? ldexpf(a.scale, -lift[u]) : lower;
    if (slice.used == 1) {
      store_rows<DT, D>(own, a.d, acc[u], scale, static_cast<T*>(second ? a.dk : a.dv) + at * a.d,
                        static_cast<uint32_t>(lane % 32 * a.hkv) * a.d, keys - key);
    } else if (key + lane % 32 < keys) {
      store_rows32<D>(a.part_dkv + ((part * keys_all(a) + at + lane % 32 * a.hkv) * 2 + second) * a.d, a.d, acc[u], scale);
    }
  }
}

// Sums of the parts of both kernels' walks, in their order, four elements a thread, bound
// by latency, 7 us:
// workgroups for rows, then workgroups for runs of `group` keys.
__device__ __forceinline__ f32x4 sum_of(const float* parts, int64_t step, int used) {
  f32x4 sum{};
  for (int k0 = 0; k0 < used; k0 += kPartsTurn) {
    f32x4 x[kPartsTurn];
#pragma unroll
    for (int k = 0; k < kPartsTurn; ++k) x[k] = *reinterpret_cast<const f32x4*>(parts + min(k0 + k, used - 1) * step);
#pragma unroll
    for (int k = 0; k < kPartsTurn; ++k)
      if (k0 + k < used) sum += x[k];
  }
  return sum;
}
template <int DT>
__global__ __launch_bounds__(kThreads) void attn_sums_kernel(const Args a, Divisor by_joins_q, Divisor by_joins_k, int q_groups, int group,
                                                             Divisor by_place_k, int tiles_first_k) {
  using T = typename Mma<DT>::T;
  using V4 = typename Mma<DT>::V4;
  const bool keys = static_cast<int>(blockIdx.x) >= q_groups;
  const int id = static_cast<int>(blockIdx.x) - (keys ? q_groups : 0), rest = a.by_hkv.divide(id), hk = id - rest * a.hkv;
  const Divisor& by = keys ? by_joins_k : by_joins_q;
  const int place = by.divide(rest), i = (rest - place * static_cast<int>(by.n)) * kThreads + static_cast<int>(threadIdx.x);
  const int of = a.by_quads.divide(i), c = (i - of * static_cast<int>(a.by_quads.n)) * 4;
  Seq s;
  int tile;
  if (!keys) {
    if (!find(a, false, a.g, kRowsGroup, place, s, tile)) return;
    const int rows = s.nq * a.g, first = tile * kRowsGroup, row = first + of;
    if (of >= kRowsGroup || row >= rows) return;
    const int used = slice_of(keys_of_group(a, s, first, rows), kKeys, a.parts, 0).used;
    if (used == 1) return;
    const int pos = a.by_g.divide(row);
    const int64_t at = ((s.b * a.rows_q + s.q0 + pos) * a.hq + hk * a.g + row - pos * a.g) * a.d + c;
    *reinterpret_cast<V4*>(static_cast<T*>(a.dq) + at) = __builtin_convertvector(sum_of(a.part_dq + at, rows_all(a) * a.d, used), V4);
    return;
  }
  Args b = a;
  b.by_place = by_place_k;
  b.tiles_first = tiles_first_k;
  if (!find(b, true, 1, group, place, s, tile)) return;
  const int all = a.cu_k ? s.nk : static_cast<int>(a.rows_k), first = tile * group, key = first + of;
  if (of >= group || key >= all) return;
  const int used = slice_of(rows_of_keys(a, s, first, group), kRowsPass, a.parts_dkv, 0).used;
  if (used == 1) return;
  const int64_t at = (s.b * a.rows_k + s.k0 + key) * a.hkv + hk, step = keys_all(a) * 2 * a.d;
  const float* p = a.part_dkv + at * 2 * a.d + c;
  *reinterpret_cast<V4*>(static_cast<T*>(a.dv) + at * a.d + c) = __builtin_convertvector(sum_of(p, step, used), V4);
  *reinterpret_cast<V4*>(static_cast<T*>(a.dk) + at * a.d + c) = __builtin_convertvector(sum_of(p + a.d, step, used), V4);
}

// ---------------------------------------------------------------- host side
int check(const fewbit_attn* a) {
  if (!a) return FEWBIT_E_NULL;
  if (a->dtype != FEWBIT_F16 && a->dtype != FEWBIT_BF16) return FEWBIT_E_DTYPE;
  if (a->reserved != 0 || a->heads_q < 1 || a->heads_kv < 1 || a->heads_q % a->heads_kv != 0) return FEWBIT_E_INVALID;
  if (a->head_dim < 8 || a->head_dim > 128 || a->head_dim % 8 != 0) return FEWBIT_E_INVALID;
  if ((a->causal != 0 && a->causal != 1) || a->window < 0 || (a->window > 0 && !a->causal)) return FEWBIT_E_INVALID;
  if (!(a->scale > 0.0f && std::isfinite(a->scale))) return FEWBIT_E_INVALID;
  constexpr int64_t kMost = int64_t{1} << 30;
  if (a->batch < 0 || a->batch >= kMost || a->rows_q < 0 || a->rows_k < 0 || a->rows_k >= kMost || a->heads_q >= 1 << 20 ||
      a->rows_q >= kMost / (a->heads_q / a->heads_kv))
    return FEWBIT_E_INVALID;
  // no more elements than there are addresses: all products of sizes below fit 64 bits
  const double seqs = a->cu_q ? 1.0 : static_cast<double>(a->batch), most = 0x1p47;
  if (seqs * a->rows_q * a->heads_q * a->head_dim >= most || seqs * a->rows_k * a->heads_kv * a->head_dim >= most) return FEWBIT_E_INVALID;
  if ((a->cu_q == nullptr) != (a->cu_k == nullptr) || (a->cu_q && a->k_len)) return FEWBIT_E_INVALID;
  return FEWBIT_OK;
}

// Rows start at multiples of 16 bytes, in ascending order: lanes' offsets inside a load have
// no sign.  Packed sequences have no stride of their own.
int check_strides(const fewbit_attn* a, const int64_t (&s)[3]) {
  const int64_t first = a->cu_q ? 0 : s[0];
  if (first < 0 || s[1] < 0 || s[2] < 0) return FEWBIT_E_INVALID;
  return first % 8 == 0 && s[1] % 8 == 0 && s[2] % 8 == 0 ? FEWBIT_OK : FEWBIT_E_ALIGN;
}

int64_t over(int64_t n, int64_t per) { return (n + per - 1) / per; }

// Places for tiles of `per` rows: exact, or for packed sequences as many as any
// division into batch (and one for the rows past the last) can need.
int64_t places_of(const fewbit_attn* a, int64_t rows, int64_t per) {
  return a->cu_q ? over(rows, per) + a->batch + 1 : over(rows, per) * a->batch;
}

// The forward that splits keys: shares per key head (0: the kernel for many rows), passes
// of a share at least, and whether no unit is in two shares, as far as the host can tell.
// It takes at most 32 rows to a sequence and key head.  One row on 64 caches of up to 8192
// keys, 16 heads to 4: 105 us, the kernel for many rows 166; on 1 of 777, 12 heads: 10 and 10; but 16
// rows on 8 of 4096, 16 heads to 4: 40 (32 rows at a time) and 21.
struct Shares {
  int64_t n, least;
  bool whole;
};
Shares shares_of(const fewbit_attn* a) {
  const int64_t rows = a->rows_q * (a->heads_q / a->heads_kv);
  if (a->cu_q || a->batch == 0 || rows == 0 || rows > kRowsWave || a->rows_k == 0) return {};
  const int64_t cus = device_cus(), passes = a->batch * over(a->rows_k + 31, kKeysSplit);
  if (a->batch >= int64_t{1} << 24 || passes >= int64_t{1} << 31) return {};
  // Every workgroup here reads the lengths of all sequences, and so does the join's for every
  // row.  Where a CU gets four sequences and key heads the tiled kernel, a workgroup to each,
  // ends as evenly: one row on 256, 1024, 4096 and 16384 caches of up to 1024, 512, 256 and 128
  // keys, 16 heads to 4 of 128: 69, 137, 301 and 819 us, here 74, 202, 1171 and 13871; on 128 of
  // up to 4096 129, here 110.
  if (a->k_len && a->batch * a->heads_kv >= 4 * cus) return {};
  // As many workgroups as the chip holds at once, or as it has CUs where that leaves one
  // pass to each (one row on 16000 keys, 16 heads to 4: 20 us in 504 workgroups, 17 in 252);
  // units of four passes are not worth a join (300 keys, 12 heads: 8.9 us joined, 7.1 whole).
  const int64_t lo = a->window ? std::max<int64_t>(0, a->rows_k - a->rows_q + 1 - a->window) / 32 * 32 : 0;
  const int64_t each = std::max<int64_t>(1, over(a->rows_k - lo, kKeysSplit));         // passes of a unit
  const auto per = [&](int64_t groups) { return over(passes, std::max<int64_t>(1, groups / a->heads_kv)); };
  Shares r;
  r.least = std::max(std::min<int64_t>(2, per(cus)), each <= 4 ? each : 1);
  r.n = over(passes, std::max(r.least, per((a->head_dim <= 64 ? 3 : 2) * cus)));
  r.whole = !a->k_len && std::max(r.least, over(each * a->batch, r.n)) % each == 0;
  // a workgroup of the join takes a row; rows that are too many for it go to the tiled kernel
  if (!fits_launch(r.n * a->heads_kv, kThreads) || (!r.whole && !fits_launch(a->batch * a->heads_kv * rows, kThreads))) return {};
  return r;
}

// The order of `tiles` tiles of every sequence.  Where walks differ in length and a CU gets
// few of them the longest come first, else a sequence's tiles follow each other: 16 x 2048
// rows, 16 heads of 128, causal, 4096 workgroups: the forward 388 us longest first, 365 so,
// with 2.4 and 0.41 GB read past the L2 (dK and dV 846 and 811, and written 0.48 and 0.27);
// 21 x 455 rows, 48 heads to 12, 1008 workgroups, dK and dV: 186 us longest first, 244 so.
void set_order(Args& r, const fewbit_attn* a, int64_t tiles) {
  r.tiles = static_cast<int>(tiles);
  r.tiles_first = a->causal && !a->window && tiles * a->batch * a->heads_kv < 12 * static_cast<int64_t>(device_cus());
  r.by_place = divisor(static_cast<int>(std::max<int64_t>(1, r.tiles_first ? a->batch : tiles)));
}

// Parts of every workgroup's walk of `passes` passes at most: as many as give every CU a
// workgroup (under a causal mask two, for the walks' lengths differ), where that shortens
// the walk by enough to pay for the join's launch and traffic, eight passes.  Forward and
// backward in a row, one and divided: 2 sequences of 2352 rows and 1 head, 38 workgroups of
// 37 passes, 191 and 96 us; 2 of 807 and 16 heads, causal, 224 workgroups of 13, 84 and 106 us
// in two parts each, which the rule leaves whole.
int64_t parts_of(int64_t groups, int64_t passes, int64_t cus, bool uneven) {
  const int64_t parts = std::min({(uneven ? 2 * cus : cus) / std::max<int64_t>(groups, 1), passes / kPassesPart, int64_t{kPartsMost}});
  return parts > 1 && passes - over(passes, parts) >= 8 ? parts : 1;
}

// Keys of a workgroup of the kernel for dK and dV: four runs of 64 where two of 32 and
// their gradients fit a wave's registers and that leaves every second CU a workgroup, else
// of 32 (3 packed sequences of 465 on average, 16 heads of 64, causal, forward and
// backward, 96 workgroups of 256 keys: 59 us, of 128: 50 us).
int64_t keys_dkv(const fewbit_attn* a) {
  const int64_t most = kPairs * 64;
  return a->head_dim <= 64 && 2 * places_of(a, a->rows_k, most) * a->heads_kv > device_cus() ? most : most / 2;
}

// Workgroups of the kernels, and parts of their walks.
struct Grid {
  int64_t q_places, k_places, parts, parts_dkv;
};
Grid grid_of(const fewbit_attn* a, bool back) {
  const int64_t g = a->heads_q / a->heads_kv, cus = device_cus();
  Grid r{places_of(a, a->rows_q * g, kRowsGroup), places_of(a, a->rows_k, keys_dkv(a)), 1, 1};
  const int64_t seqs = a->cu_q ? std::max<int64_t>(a->batch, 1) : 1;              // packed: lengths are not known here
  const int64_t keys = a->rows_k / seqs, rows = a->rows_q * g / seqs;
  const bool uneven = a->causal && !a->window && 2 * a->rows_q > a->rows_k;
  const int64_t seen = a->window ? std::min<int64_t>(keys, int64_t{a->window} + kRowsGroup / g) : keys;
  const int64_t seers = a->window ? std::min(rows, (a->window + keys_dkv(a)) * g) : rows;
  r.parts = parts_of(r.q_places * a->heads_kv, over(seen, kKeys), cus, uneven);
  if (back) r.parts_dkv = parts_of(r.k_places * a->heads_kv, over(seers, kRowsPass), cus, uneven);
  return r;
}

Args args_of(const fewbit_attn* a) {
  Args r{};
  r.cu_q = a->cu_q;
  r.cu_k = a->cu_k;
  r.k_len = a->k_len;
  for (int i = 0; i < 3; ++i) {
    r.qs[i] = a->q_stride[i];
    r.ks[i] = a->k_stride[i];
    r.vs[i] = a->v_stride[i];
    r.ds[i] = a->dout_stride[i];
  }
  r.rows_q = a->rows_q;
  r.rows_k = a->rows_k;
  r.batch = static_cast<int>(a->batch);
  r.hq = a->heads_q;
  r.hkv = a->heads_kv;
  r.g = a->heads_q / a->heads_kv;
  r.d = a->head_dim;
  r.causal = a->causal;
  r.window = std::min(a->window, 1 << 30);
  r.scale = a->scale;
  r.by_g = divisor(r.g);
  r.by_hkv = divisor(r.hkv);
  r.by_parts = r.by_parts_dkv = divisor(1);
  r.by_quads = divisor(r.d / 4);
  return r;
}

int64_t rounded(int64_t n) { return over(n, 4) * 4; }         // floats, to whole 16 bytes

#define FEWBIT_ATTN_START(KERNEL, ARGS, GROUPS, STREAM)                                                              \
  ((ARGS).d <= 64 ? (bf16 ? launch(KERNEL<FEWBIT_BF16, 64>, dim3(static_cast<unsigned>(GROUPS)), kThreads, STREAM, ARGS)    \
                          : launch(KERNEL<FEWBIT_F16, 64>, dim3(static_cast<unsigned>(GROUPS)), kThreads, STREAM, ARGS))    \
                  : (bf16 ? launch(KERNEL<FEWBIT_BF16, 128>, dim3(static_cast<unsigned>(GROUPS)), kThreads, STREAM, ARGS)   \
                          : launch(KERNEL<FEWBIT_F16, 128>, dim3(static_cast<unsigned>(GROUPS)), kThreads, STREAM, ARGS)))

hipError_t start_split(const Args& r, bool bf16, unsigned groups, hipStream_t st) {
  return r.d <= 64 ? launch(bf16 ? attn_split_kernel<FEWBIT_BF16, 64> : attn_split_kernel<FEWBIT_F16, 64>, dim3(groups), kThreads, st, r)
                   : launch(bf16 ? attn_split_kernel<FEWBIT_BF16, 128> : attn_split_kernel<FEWBIT_F16, 128>, dim3(groups), kThreads, st, r);
}

template <int D, int SUBS>
hipError_t start_dkv(const Args& r, bool bf16, unsigned groups, hipStream_t st) {
  return launch(bf16 ? attn_dkv_kernel<FEWBIT_BF16, D, SUBS> : attn_dkv_kernel<FEWBIT_F16, D, SUBS>, dim3(groups), kThreadsPairs, st, r);
}

}  // namespace

extern "C" int64_t fewbit_attn_workspace(const fewbit_attn* a, int32_t backward) {
  const int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  const int64_t rows = (a->cu_q ? 1 : a->batch) * a->rows_q * a->heads_q;
  const Grid g = grid_of(a, backward != 0);
  if (backward) {
    const int64_t keys = (a->cu_q ? 1 : a->batch) * a->rows_k * a->heads_kv;
    return (2 * rounded(rows) + (g.parts > 1 ? g.parts * rows * a->head_dim : 0) + (g.parts_dkv > 1 ? g.parts_dkv * keys * 2 * a->head_dim : 0)) *
           static_cast<int64_t>(sizeof(float));
  }
  const int64_t shares = shares_of(a).n, of = a->rows_q * (a->heads_q / a->heads_kv);
  const int64_t left = shares > 0 ? (shares + a->batch) * a->heads_kv * of : g.parts > 1 ? g.parts * rows : 0;
  return left * (a->head_dim + 1) * static_cast<int64_t>(sizeof(float));
}

extern "C" int fewbit_attn_fwd(const fewbit_attn* a, const void* q, const void* k, const void* v, void* out, float* lse,
                               void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  if (a->batch == 0 && a->cu_q == nullptr) return FEWBIT_OK;
  if (a->rows_q == 0) return FEWBIT_OK;
  if (!q || !out || !lse || (a->rows_k > 0 && (!k || !v))) return FEWBIT_E_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out)) return FEWBIT_E_ALIGN;
  for (const auto* s : {&a->q_stride, &a->k_stride, &a->v_stride}) {
    rc = check_strides(a, *s);
    if (rc != FEWBIT_OK) return rc;
  }
  const int64_t need = fewbit_attn_workspace(a, 0);
  if (need > 0 && !workspace) return FEWBIT_E_NULL;
  if (workspace_bytes < need) return FEWBIT_E_INVALID;
  if (need > 0 && misaligned(workspace)) return FEWBIT_E_ALIGN;
  const bool bf16 = a->dtype == FEWBIT_BF16;
  Args r = args_of(a);
  r.q = q;
  r.k = k;
  r.v = v;
  r.o = out;
  r.lse = lse;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t rows = a->rows_q * r.g;
  const Shares shares = shares_of(a);
  r.shares = static_cast<int>(shares.n);
  r.share_least = static_cast<int>(shares.least);
  if (r.shares == 0) {
    const Grid g = grid_of(a, false);
    set_order(r, a, over(rows, kRowsGroup));
    r.parts = static_cast<int>(g.parts);
    r.by_parts = divisor(r.parts);
    if (r.parts > 1) {
      r.part_o = static_cast<float*>(workspace);
      r.part_lse = r.part_o + g.parts * (a->cu_q ? 1 : a->batch) * a->rows_q * r.hq * r.d;
    }
    const int64_t share = over(int64_t{kRowsGroup} * r.d / 4, kThreads), joins = g.q_places * r.hkv * share, groups = g.q_places * r.hkv * g.parts;
    if (!fits_launch(groups, kThreads) || (r.parts > 1 && !fits_launch(joins, kThreads))) return FEWBIT_E_INVALID;
    rc = check_stream_device(st);
    if (rc != FEWBIT_OK) return rc;
    rc = launch_status("fewbit_attn_fwd", FEWBIT_ATTN_START(attn_fwd_kernel, r, groups, st));
    if (rc != FEWBIT_OK || r.parts == 1) return rc;
    return launch_status("fewbit_attn_fwd", launch(bf16 ? attn_parts_kernel<FEWBIT_BF16> : attn_parts_kernel<FEWBIT_F16>,
                                                   dim3(static_cast<unsigned>(joins)), kThreads, st, r, divisor(static_cast<int>(share))));
  }
  r.part_o = static_cast<float*>(workspace);
  r.rows = static_cast<int>(rows);
  r.by_rows = divisor(r.rows);
  r.part_lse = r.part_o + (r.shares + a->batch) * r.hkv * r.rows * r.d;
  const int64_t groups = static_cast<int64_t>(r.shares) * r.hkv, joins = a->batch * r.hkv * r.rows;       // both fit a launch
  rc = check_stream_device(st);
  if (rc != FEWBIT_OK) return rc;
  rc = launch_status("fewbit_attn_fwd", start_split(r, bf16, static_cast<unsigned>(groups), st));
  if (rc != FEWBIT_OK || shares.whole) return rc;
  return launch_status("fewbit_attn_fwd", launch(bf16 ? attn_join_kernel<FEWBIT_BF16> : attn_join_kernel<FEWBIT_F16>,
                                                 dim3(static_cast<unsigned>(joins)), kThreads, st, r));
}

extern "C" int fewbit_attn_bwd(const fewbit_attn* a, const void* dout, const void* q, const void* k, const void* v,
                               const void* out, const float* lse, void* dq, void* dk, void* dv, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  int rc = check(a);
  if (rc != FEWBIT_OK) return rc;
  if ((a->batch == 0 && a->cu_q == nullptr) || (a->rows_q == 0 && a->rows_k == 0)) return FEWBIT_OK;
  if (a->rows_q > 0 && (!q || !dout || !out || !lse || !dq || !workspace)) return FEWBIT_E_NULL;
  if (a->rows_k > 0 && (!k || !v || !dk || !dv)) return FEWBIT_E_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(dout) || misaligned(dq) ||
      misaligned(dk) || misaligned(dv))
    return FEWBIT_E_ALIGN;
  for (const auto* s : {&a->q_stride, &a->k_stride, &a->v_stride, &a->dout_stride}) {
    rc = check_strides(a, *s);
    if (rc != FEWBIT_OK) return rc;
  }
  if (workspace_bytes < fewbit_attn_workspace(a, 1)) return FEWBIT_E_INVALID;
  const bool bf16 = a->dtype == FEWBIT_BF16;
  Args r = args_of(a);
  const Grid g = grid_of(a, true);
  const int group = static_cast<int>(keys_dkv(a));
  const bool join_q = g.parts > 1 && a->rows_q > 0, join_k = g.parts_dkv > 1 && a->rows_k > 0;
  const int64_t share_q = over(int64_t{kRowsGroup} * r.d / 4, kThreads), share_k = over(int64_t{group} * r.d / 4, kThreads);
  const int64_t joins_q = join_q ? g.q_places * r.hkv * share_q : 0, joins_k = join_k ? g.k_places * r.hkv * share_k : 0;
  const int64_t q_groups = g.q_places * r.hkv * g.parts, k_groups = g.k_places * r.hkv * g.parts_dkv;
  if (!fits_launch(q_groups, kThreads) || !fits_launch(k_groups, kThreadsPairs) || !fits_launch(joins_q + joins_k, kThreads))
    return FEWBIT_E_INVALID;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  rc = check_stream_device(st);
  if (rc != FEWBIT_OK) return rc;
  r.q = q;
  r.k = k;
  r.v = v;
  r.out = out;
  r.dout = dout;
  r.lse = const_cast<float*>(lse);
  r.stats = static_cast<float*>(workspace);
  const int64_t rows_all = (a->cu_q ? 1 : a->batch) * a->rows_q * a->heads_q;
  r.stats_delta = rounded(rows_all);
  r.dq = dq;
  r.dk = dk;
  r.dv = dv;
  r.parts = static_cast<int>(g.parts);
  r.parts_dkv = static_cast<int>(g.parts_dkv);
  r.by_parts = divisor(r.parts);
  r.by_parts_dkv = divisor(r.parts_dkv);
  r.part_dq = r.stats + 2 * r.stats_delta;
  r.part_dkv = r.part_dq + (g.parts > 1 ? g.parts * rows_all * r.d : 0);
  const int64_t tiles_q = over(a->rows_q * r.g, kRowsGroup), tiles_k = over(a->rows_k, group);
  if (a->rows_q > 0) {
    set_order(r, a, tiles_q);
    rc = launch_status("fewbit_attn_bwd", FEWBIT_ATTN_START(attn_dq_kernel, r, q_groups, st));
    if (rc != FEWBIT_OK) return rc;
  }
  if (a->rows_k > 0) {
    set_order(r, a, tiles_k);
    const auto start = r.d > 64 ? start_dkv<128, 1> : group == kPairs * 64 ? start_dkv<64, 2> : start_dkv<64, 1>;
    rc = launch_status("fewbit_attn_bwd", start(r, bf16, static_cast<unsigned>(k_groups), st));
  }
  if (rc != FEWBIT_OK || (!join_q && !join_k)) return rc;
  Args r_k = r;
  set_order(r, a, tiles_q);
  set_order(r_k, a, tiles_k);
  return launch_status("fewbit_attn_bwd",
                       launch(bf16 ? attn_sums_kernel<FEWBIT_BF16> : attn_sums_kernel<FEWBIT_F16>, dim3(static_cast<unsigned>(joins_q + joins_k)),
                              kThreads, st, r, divisor(static_cast<int>(share_q)), divisor(static_cast<int>(share_k)), static_cast<int>(joins_q),
                              group, r_k.by_place, r_k.tiles_first));
}
