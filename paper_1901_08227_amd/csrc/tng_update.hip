// Matrices orthogonalised by Newton-Schulz products on the matrix units (gfx950).
//
//   X = x / (||x|| + eps);  a step: G = X X^T,  P = a + b G + c G G,  X' = P X
//
// with X lying so that it has no more rows n than columns m.  G and P are symmetric: only half of them is computed.
//
// Numbers are held as pairs of binary16, v = high + low with low = v - high rounded: 22 bits of v and more, as long as low is no subnormal number, for
// which v is held times a power of two.  A product of pairs is three products, high high + high low + low high (low low is below the last bit), summed
// in binary32.  That is as exact as binary32 within a factor of two, and three times the work at sixteen times the rate.  Bits of 16 alone would not do: what rounding
// takes from a direction of small singular value grows with it, by 3.4 a step.
#include "tng_layer_device.hpp"
#include "tng_pair_loads.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace tng {
namespace {

typedef f16_t v4h __attribute__((ext_vector_type(4)));
typedef f16_t v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

// What is held is v times these: with singular values of X below 2 and of P below 8 no pair leaves binary16, and of a number of 2^-17 every bit counts.
constexpr float kOfX = 0x1p14f, kOfGram = 0x1p14f, kOfPoly = 0x1p13f;

// A matrix of pairs: rows of blocks of 32 columns, 128 bytes each: the high parts, then the low parts.  What lies between the last column and the end of
// its block is 0.
constexpr uint32_t kBlockCols = 32;
constexpr uint64_t kBlockBytes = 128;
inline uint64_t pair_row(uint64_t cols) { return (cols + kBlockCols - 1) / kBlockCols * kBlockBytes; }

struct Pairs {
  char* p;
  uint64_t ld, pitch;  // bytes from row to row, and from matrix to matrix
};
__host__ __device__ inline uint64_t pair_at(uint64_t col) { return col / kBlockCols * kBlockBytes + col % kBlockCols * 2; }

__device__ __forceinline__ void split(float v, f16_t& high, f16_t& low) {
  high = (f16_t)v;
  low = (f16_t)(v - (float)high);
}

// ---- ||x||, and x as pairs both ways round

struct StartTask {
  uint64_t rows, cols;  // of x as it lies
  View x;
  double* part;  // [matrix][parts]
  uint32_t parts;
  float eps;
  bool tall;       // x has more rows than columns: X is x turned
  Pairs x_by_n, x_by_m;  // X and X turned
};

// Squares are summed in binary64, which holds those of every number; a matrix's parts in a fixed order.
template <typename T>
__global__ void __launch_bounds__(kBlock) squares_kernel(StartTask p) {
  __shared__ double of_wave[kBlock / kWave];
  const uint32_t m = blockIdx.y;
  const T* x = static_cast<const T*>(p.x.p) + m * p.x.pitch;
  double sum = 0.;
  // (a workgroup's rows, a piece of a row for each of its wavefronts at a time)
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint64_t pieces = (p.cols + kWave * 8 - 1) / (kWave * 8), all = p.rows * pieces;
  for (uint64_t k = (uint64_t)blockIdx.x * (kBlock / kWave) + wave; k < all; k += (uint64_t)p.parts * (kBlock / kWave)) {
    const uint64_t r = k / pieces, c = (k - r * pieces) * (kWave * 8) + lane * 8;
    if (c >= p.cols) continue;
    float v[8];
    load_n_within<T, 8>(x + r * p.x.ld + c, p.cols - c, 0.f, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += (double)v[i] * (double)v[i];
  }
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  if (lane == 0) of_wave[wave] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  sum = 0.;
  for (int k = 0; k < kBlock / kWave; ++k) sum += of_wave[k];
  p.part[(uint64_t)m * p.parts + blockIdx.x] = sum;
}

__device__ __forceinline__ double sum_of_parts(const double* part, uint32_t parts, uint32_t lane) {
  double sum = 0.;
  for (uint32_t k = lane; k < parts; k += kWave) sum += part[k];
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  return sum;
}
// What x is multiplied by, from its squares.  (A matrix that holds what is not finite is NaN as a whole.)
__device__ __forceinline__ double inverse_of(double squares, float eps) {
  return (squares < __builtin_inf() ? 1. / (sqrt(squares) + (double)eps) : __builtin_nan("")) * (double)kOfX;
}

// 64 x 64 elements of x for a workgroup: as pairs along the columns, and turned, along the rows.
constexpr uint32_t kTurn = 64;

template <typename T>
__global__ void __launch_bounds__(kBlock) start_kernel(StartTask p) {
  __shared__ uint32_t tile[kTurn][kTurn + 1];  // [row][column]: a pair
  __shared__ double inverse;
  const uint32_t m = blockIdx.z;
  if (threadIdx.x < kWave) {
    const double sum = sum_of_parts(p.part + (uint64_t)m * p.parts, p.parts, threadIdx.x);
    if (threadIdx.x == 0) inverse = inverse_of(sum, p.eps);
  }
  __syncthreads();
  const double inv = inverse;
  const T* x = static_cast<const T*>(p.x.p) + m * p.x.pitch;
  const uint64_t r0 = (uint64_t)blockIdx.y * kTurn, c0 = (uint64_t)blockIdx.x * kTurn;
  const Pairs along = p.tall ? p.x_by_m : p.x_by_n, turned = p.tall ? p.x_by_n : p.x_by_m;
  const uint32_t eight = threadIdx.x % 8, line = threadIdx.x / 8;
  auto put = [&](const Pairs& to, uint64_t row, uint64_t col, const uint32_t (&pair)[8]) {
    v8h high, low;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      high[i] = __builtin_bit_cast(f16_t, (uint16_t)pair[i]);
      low[i] = __builtin_bit_cast(f16_t, (uint16_t)(pair[i] >> 16));
    }
    char* at = to.p + m * to.pitch + row * to.ld + pair_at(col);
    *reinterpret_cast<v8h*>(at) = high;
    *reinterpret_cast<v8h*>(at + 64) = low;
  };
#pragma unroll
  for (uint32_t k = 0; k < kTurn; k += kBlock / 8) {
    const uint64_t r = r0 + k + line, c = c0 + eight * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (r < p.rows && c < p.cols) load_n_within<T, 8>(x + r * p.x.ld + c, p.cols - c, 0.f, v);
    uint32_t pair[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f16_t high, low;
      split(r < p.rows && c + i < p.cols ? (float)((double)v[i] * inv) : 0.f, high, low);
      pair[i] = (uint32_t)__builtin_bit_cast(uint16_t, high) | (uint32_t)__builtin_bit_cast(uint16_t, low) << 16;
      tile[k + line][eight * 8 + i] = pair[i];
    }
    if (r < p.rows && c < (p.cols + kBlockCols - 1) / kBlockCols * kBlockCols) put(along, r, c, pair);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < kTurn; k += kBlock / 8) {
    const uint64_t c = c0 + k + line, r = r0 + eight * 8;
    uint32_t pair[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pair[i] = tile[eight * 8 + i][k + line];
    if (c < p.cols && r < (p.rows + kBlockCols - 1) / kBlockCols * kBlockCols) put(turned, c, r, pair);
  }
}

// ---- products of pairs: result (r, c) is the sum over k of a(r, k) b(c, k)

// What becomes of the sums.
constexpr int kGram = 0, kPoly = 1, kApply = 2, kLast = 3;

struct PairTask {
  uint32_t rows, cols, stages;  // rows of a, of b; blocks of 32 that they are long
  uint32_t planes;
  Pairs a, b;
  Pairs gram;               // kPoly
  float plus, times, square;  // kPoly: a, b, c
  Pairs by_r, by_c;         // results as rows of r, and turned, as rows of c
  View y;                   // kLast: rows of c
  float scale;
  uint32_t full, splits;  // tiles before number `full` are made whole, the others by `splits` workgroups each, and joined
  float* part;            // [tile from full on][split][kRows kCols]
};

// The tile of a number, in columns of kGroup tiles of rows, which are about square; HALF: only tiles with c <= r.
struct Place {
  uint32_t r, c;
};
template <bool HALF>
__device__ __forceinline__ Place place_of(uint32_t number, uint32_t down, uint32_t across) {
  constexpr uint32_t kGroup = 8;
  if (!HALF) {
    const uint32_t group = number / (kGroup * across), first = group * kGroup, high = min(kGroup, down - first), in = number - group * kGroup * across;
    return Place{first + in % high, in / high};
  }
  uint32_t first = 0;
  for (;;) {
    const uint32_t high = min(kGroup, down - first), count = high * first + high * (high + 1) / 2;
    if (number < count) {
      if (number < high * first) return Place{first + number % high, number / high};
      number -= high * first;
      uint32_t c = 0;
      while (number >= high - c) number -= high - c++;
      return Place{first + c + number, first + c};
    }
    number -= count;
    first += kGroup;
  }
}
inline uint32_t tiles_of(bool half, uint32_t down, uint32_t across) { return half ? down * (down + 1) / 2 : down * across; }

// Workgroups go to the eight dies in turn: each die takes a run of tiles that lie together.
__device__ __forceinline__ uint32_t number_of(uint32_t block, uint32_t all) {
  constexpr uint32_t kDies = 8;
  const uint32_t die = block % kDies, each = all / kDies, more = all % kDies;
  return die * each + min(die, more) + block / kDies;
}

constexpr uint32_t turn_pitch(int tiles) { return tiles * 16 + 4; }

// A wavefront makes RN x CN tiles of 16 x 16 results, WR x WC of them a workgroup's tile.  A stage is 32 columns of the operands' rows, 128 bytes each; SLOTS of them lie
// in LDS.  While the products of a stage run, the next one's fragments are read into registers, and the loads of the stage that follows the last one in LDS
// are asked for, in the place of the one that has been read: one wait and one barrier a stage.  Tiles of 128 take 0.55 us a stage, those of 64, two
// on a CU, 0.34: the loads, of 32 and 16 KB a tile and stage out of the die's cache.  Tiles of 128 by four wavefronts, two on a CU, take 1.1, as long, but one
// tile's beginning and end pass while the other is multiplied: 4 x 2053 x 1003 748 -> 703 us, 100 x 256 x 256 357 -> 317.  (A meeting every other stage, with five in
// LDS: no sooner.)
template <int RN, int CN, int WR, int WC, int SLOTS>
struct PairKernel {
  static constexpr int kRows = RN * WR * 16, kCols = CN * WC * 16, kWaves = WR * WC, kThreads = kWaves * kWave;
  static constexpr int kStageBytes = (kRows + kCols) * 128, kRing = SLOTS * kStageBytes;
  static constexpr int kLoads = (kRows + kCols) / 8 / kWaves, kLoadsOfA = kRows / 8 / kWaves;
  static_assert(kRows % (8 * kWaves) == 0 && kCols % (8 * kWaves) == 0, "loads divide evenly");
  // Behind the stages: the results of 32 rows of each wavefront at a time, turned.  (Four words more a row: a wavefront's four groups of rows meet in no bank.)
  static constexpr int kTurnBytes = 32 * turn_pitch(CN) * 4;
  static_assert(RN % 2 == 0 && kTurnBytes * kWaves <= kRing, "results are turned in the stages' place");
};

// What becomes of two tiles of rows, from r_first on, of a wavefront's results; turn: its place in LDS.  both: results go both ways round.
template <typename T, int END, int CN>
__device__ __forceinline__ void finish_rows(const PairTask& p, uint32_t plane, bool both, uint32_t r_first, uint32_t c_first, const v4f (&sum)[2][CN],
                                            uint32_t* turn, uint32_t lane) {
  constexpr uint32_t kPitch = turn_pitch(CN);
  // A lane has four results of consecutive r for one c.
  const uint32_t i = lane % 16, r_in = r_first + lane / 16 * 4, c_in = c_first + i;
  const uint32_t end_r = (p.rows + kBlockCols - 1) / kBlockCols * kBlockCols, end_c = (p.cols + kBlockCols - 1) / kBlockCols * kBlockCols;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < CN; ++b) {
      const uint32_t r = r_in + a * 16, c = c_in + b * 16;
      float v[4];
      if (END == kLast) {
        if (r >= p.rows || c >= p.cols) continue;
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = sum[a][b][n] * (1.f / (kOfPoly * kOfX)) * p.scale;
        store_n_within<T, 4>(static_cast<T*>(p.y.p) + plane * p.y.pitch + c * p.y.ld + r, p.rows - r, v);
        continue;
      }
      const bool in = c < p.cols && r < end_r;
      if (END == kPoly) {
        v4h g_high = {}, g_low = {};
        if (in) {
          const char* at = p.gram.p + plane * p.gram.pitch + c * p.gram.ld + pair_at(r);
          g_high = *reinterpret_cast<const v4h*>(at);
          g_low = *reinterpret_cast<const v4h*>(at + 64);
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const float gram = ((float)g_high[n] + (float)g_low[n]) * (1.f / kOfGram), square = sum[a][b][n] * (1.f / (kOfGram * kOfGram));
          v[n] = (p.times * gram + p.square * square + (r + n == c ? p.plus : 0.f)) * kOfPoly;
        }
      } else {
        constexpr float kUnit = END == kGram ? kOfGram / (kOfX * kOfX) : kOfX / (kOfPoly * kOfX);
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = sum[a][b][n] * kUnit;
      }
      v4h high, low;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        f16_t h, l;
        split(r + n < p.rows && c < p.cols ? v[n] : 0.f, h, l);
        high[n] = h;
        low[n] = l;
        if (both)
          turn[(a * 16 + lane / 16 * 4 + n) * kPitch + b * 16 + i] =
              (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
      }
      if (in) {
        char* at = p.by_c.p + plane * p.by_c.pitch + c * p.by_c.ld + pair_at(r);
        *reinterpret_cast<v4h*>(at) = high;
        *reinterpret_cast<v4h*>(at + 64) = low;
      }
    }
  if (END == kLast || !both) return;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wavefront's own: what its lanes have written is there)
  constexpr uint32_t kEights = CN * 2;                // of a row
  static_assert(32 * kEights % kWave == 0, "a row's eights are divided evenly");
#pragma unroll
  for (uint32_t piece = 0; piece < 32 * kEights; piece += kWave) {
    const uint32_t row = (piece + lane) / kEights, eight = (piece + lane) % kEights, r = r_first + row, c = c_first + eight * 8;
    const uint32_t* from = turn + row * kPitch + eight * 8;
    typedef uint32_t four __attribute__((ext_vector_type(4)));
    const four w0 = *reinterpret_cast<const four*>(from), w1 = *reinterpret_cast<const four*>(from + 4);
    four high, low;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      high[n] = __builtin_amdgcn_perm(w0[2 * n + 1], w0[2 * n], 0x05040100u);
      low[n] = __builtin_amdgcn_perm(w0[2 * n + 1], w0[2 * n], 0x07060302u);
      high[n + 2] = __builtin_amdgcn_perm(w1[2 * n + 1], w1[2 * n], 0x05040100u);
      low[n + 2] = __builtin_amdgcn_perm(w1[2 * n + 1], w1[2 * n], 0x07060302u);
    }
    if (r < p.rows && c < end_c) {
      char* at = p.by_r.p + plane * p.by_r.pitch + r * p.by_r.ld + pair_at(c);
      *reinterpret_cast<four*>(at) = high;
      *reinterpret_cast<four*>(at + 64) = low;
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// What a workgroup does: a tile, or a piece of the depth of one, whose sums go to p.part.
struct Work {
  uint32_t plane, first, stages;
  int part;  // -1: the whole tile
  Place place;
};
template <typename K, bool HALF>
__device__ __forceinline__ Work work_of(const PairTask& p) {
  const uint32_t down = (p.rows + K::kRows - 1) / K::kRows, across = (p.cols + K::kCols - 1) / K::kCols, each = HALF ? down * (down + 1) / 2 : down * across;
  Work w{0, 0, p.stages, -1, {}};
  uint32_t number;
  if (blockIdx.x < p.full) {
    number = number_of(blockIdx.x, p.full);
  } else {
    w.part = (int)(blockIdx.x - p.full);
    const uint32_t tile = (uint32_t)w.part / p.splits, s = (uint32_t)w.part - tile * p.splits;
    number = p.full + tile;
    w.first = p.stages * s / p.splits;
    w.stages = p.stages * (s + 1) / p.splits - w.first;
  }
  w.plane = number / each;
  w.place = place_of<HALF>(number - w.plane * each, down, across);
  return w;
}

// What becomes of a workgroup's sums.  lds: of the stages, which nobody reads any more.
template <typename T, int END, typename K, int RN, int CN, int WC>
__device__ __forceinline__ void finish_tile(const PairTask& p, const Work& w, const v4f (&sum)[RN][CN], char* lds, uint32_t lane, uint32_t wave) {
  if (w.part >= 0) {  // as they lie in the registers
    float* to = p.part + (uint64_t)w.part * (K::kRows * K::kCols) + wave * (RN * CN * 256) + lane * 4;
#pragma unroll
    for (int a = 0; a < RN; ++a)
#pragma unroll
      for (int b = 0; b < CN; ++b) *reinterpret_cast<v4f*>(to + (a * CN + b) * 256) = sum[a][b];
    return;
  }
  const bool both = !(END == kGram || END == kPoly) || w.place.r != w.place.c;
  uint32_t* turn = reinterpret_cast<uint32_t*>(lds + wave * K::kTurnBytes);
#pragma unroll
  for (int a = 0; a < RN; a += 2) {
    v4f two[2][CN];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int b = 0; b < CN; ++b) two[k][b] = sum[a + k][b];
    finish_rows<T, END, CN>(p, w.plane, both, w.place.r * K::kRows + (wave / WC * RN + a) * 16, w.place.c * K::kCols + wave % WC * CN * 16, two, turn, lane);
  }
}

// Pieces of a tile's depth joined, in their order, two tiles of rows of each wavefront.
template <typename T, int END, int RN, int CN, int WR, int WC>
__global__ void __launch_bounds__(WR* WC* kWave) pair_join_kernel(PairTask p) {
  using K = PairKernel<RN, CN, WR, WC, 2>;
  constexpr bool kHalf = END == kGram || END == kPoly;
  __shared__ __align__(16) char lds[K::kTurnBytes * K::kWaves];
  const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), a = blockIdx.y * 2;
  const uint32_t down = (p.rows + K::kRows - 1) / K::kRows, across = (p.cols + K::kCols - 1) / K::kCols, each = kHalf ? down * (down + 1) / 2 : down * across;
  const uint32_t number = p.full + blockIdx.x, plane = number / each;
  const Place place = place_of<kHalf>(number - plane * each, down, across);
  v4f sum[2][CN] = {};
  const float* from = p.part + (uint64_t)blockIdx.x * p.splits * (K::kRows * K::kCols) + wave * (RN * CN * 256) + a * CN * 256 + lane * 4;
  for (uint32_t s = 0; s < p.splits; ++s, from += K::kRows * K::kCols)
#pragma unroll
    for (int k = 0; k < 2 * CN; ++k) sum[k / CN][k % CN] += *reinterpret_cast<const v4f*>(from + k * 256);
  finish_rows<T, END, CN>(p, plane, !kHalf || place.r != place.c, place.r * K::kRows + (wave / WC * RN + a) * 16, place.c * K::kCols + wave % WC * CN * 16, sum,
                          reinterpret_cast<uint32_t*>(lds + wave * K::kTurnBytes), lane);
}

// A workgroup's operands: number j of a wavefront's loads takes 8 rows, a row eight lanes.  Rows behind the last one, and stages behind the last one, are out
// of bounds: nothing is read, and what the loads clear belongs to no result.
template <typename K>
struct Operands {
  PairRows a, b;
  uint32_t offset_a, offset_b, lds;
  __device__ __forceinline__ Operands(const PairTask& p, const Work& w, uint32_t lane, uint32_t wave, const char* at)
      : a(PairRows::of(reinterpret_cast<uint64_t>(p.a.p) + w.plane * p.a.pitch, p.a.ld, p.rows, w.place.r * K::kRows, K::kRows, w.first, w.stages)),
        b(PairRows::of(reinterpret_cast<uint64_t>(p.b.p) + w.plane * p.b.pitch, p.b.ld, p.cols, w.place.c * K::kCols, K::kCols, w.first, w.stages)),
        offset_a(a.offset(lane, wave)),
        offset_b(b.offset(lane, wave)),
        lds((uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)at) + wave * 1024) {}
  __device__ __forceinline__ void load(int j, uint32_t slot) const {
    const bool of_a = j < K::kLoadsOfA;
    const PairRows::Descriptor d = of_a ? a.from(j * K::kWaves * 8) : b.from((j - K::kLoadsOfA) * K::kWaves * 8);
    load_to_lds(d.base, d.bytes, of_a ? offset_a : offset_b, lds + slot + j * K::kWaves * 1024);
  }
  __device__ __forceinline__ void next() {
    a.next();
    b.next();
    a.bytes = __builtin_amdgcn_readfirstlane(a.bytes);  // (descriptors lie in scalar registers)
    b.bytes = __builtin_amdgcn_readfirstlane(b.bytes);
  }
};

// One tile of rows times the columns' tiles: three products of each pair.
template <int CN>
__device__ __forceinline__ void multiply(v4f (&sum)[CN], const v8h (&a)[2], const v8h (&b)[CN][2]) {
#pragma unroll
  for (int k = 0; k < CN; ++k) sum[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0], b[k][1], sum[k], 0, 0, 0);
#pragma unroll
  for (int k = 0; k < CN; ++k) sum[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[1], b[k][0], sum[k], 0, 0, 0);
#pragma unroll
  for (int k = 0; k < CN; ++k) sum[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0], b[k][0], sum[k], 0, 0, 0);
  __builtin_amdgcn_sched_barrier(0);
}

template <typename T, int END, int RN, int CN, int WR, int WC, int SLOTS>
__global__ void __launch_bounds__(WR* WC* kWave) pair_kernel(PairTask p) {
  using K = PairKernel<RN, CN, WR, WC, SLOTS>;
  constexpr bool kHalf = END == kGram || END == kPoly;
  __shared__ __align__(1024) char lds[K::kRing];
  const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wr = wave / WC, wc = wave % WC, i = lane % 16;
  const Work w = work_of<K, kHalf>(p);
  Operands<K> of(p, w, lane, wave, lds);
  // Where a lane reads its rows' pieces; the low parts are four pieces on.
  const uint32_t at_a = (wr * RN * 16 + i) * 128 + (lane / 16 ^ (i >> 1 & 7u)) * 16;
  const uint32_t at_b = (K::kRows + wc * CN * 16 + i) * 128 + (lane / 16 ^ (i >> 1 & 7u)) * 16;
  struct Fragments {
    v8h a[RN][2], b[CN][2];
  };
  auto read_a = [&](Fragments& f, int k, uint32_t slot) {
    f.a[k][0] = *reinterpret_cast<const v8h*>(lds + slot + at_a + k * 2048);
    f.a[k][1] = *reinterpret_cast<const v8h*>(lds + slot + (at_a ^ 64u) + k * 2048);
  };
  auto read_b = [&](Fragments& f, int k, uint32_t slot) {
    f.b[k][0] = *reinterpret_cast<const v8h*>(lds + slot + at_b + k * 2048);
    f.b[k][1] = *reinterpret_cast<const v8h*>(lds + slot + (at_b ^ 64u) + k * 2048);
  };
  v4f sum[RN][CN];
#pragma unroll
  for (int a = 0; a < RN; ++a)
#pragma unroll
    for (int b = 0; b < CN; ++b) sum[a][b] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < SLOTS; ++k) {
#pragma unroll
    for (int j = 0; j < K::kLoads; ++j) of.load(j, k * K::kStageBytes);
    of.next();
  }
  Fragments even, odd;
  wait_and_meet<(SLOTS - 1) * K::kLoads>();
#pragma unroll
  for (int k = 0; k < RN; ++k) read_a(even, k, 0);
#pragma unroll
  for (int k = 0; k < CN; ++k) read_b(even, k, 0);
  uint32_t slot = 0;
  auto stage = [&](Fragments& now, Fragments& then) {
    const uint32_t next = slot + K::kStageBytes == K::kRing ? 0u : slot + K::kStageBytes;
    wait_and_meet<(SLOTS - 2) * K::kLoads>();  // this stage is in registers everywhere, and the next one in LDS
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kReads = (CN + RN - 1) / RN, kAsks = (K::kLoads + RN - 1) / RN;
#pragma unroll
    for (int g = 0; g < RN; ++g) {
      read_a(then, g, next);
#pragma unroll
      for (int k = g * kReads; k < (g + 1) * kReads && k < CN; ++k) read_b(then, k, next);
#pragma unroll
      for (int j = g * kAsks; j < (g + 1) * kAsks && j < K::kLoads; ++j) of.load(j, slot);
      multiply<CN>(sum[g], now.a[g], now.b);
    }
    of.next();
    slot = next;
  };
  uint32_t k = 0;
  for (; k + 2 <= w.stages; k += 2) {
    stage(even, odd);
    stage(odd, even);
  }
  if (k < w.stages) stage(even, odd);
  wait_and_meet<0>();  // (the loads that found nothing are done, and LDS is read everywhere)
  finish_tile<T, END, K, RN, CN, WC>(p, w, sum, lds, lane, wave);
}

// The same with tiles whose wavefronts have no registers for a second stage's fragments of the rows: those are read two groups ahead.  Before the last two groups
// of a stage nothing of it is left in LDS to read, and all meet: the next stage is there, and the place of this one is free.  EARLY: loads after each
// of the last two groups; the others follow the first groups of the next stage.  (256 x 256 with one, two and four: 306, 288, 291 us for P X of 4096 x 4096.)
// The matrix units bound it, at the clock that their power leaves: 287 us for P X of 4096 x 4096, 1.44 PFLOP/s of products of 16 bits, 72 % of the units' time at
// 1.88 GHz (the library's product of binary16 makes 1.26 there); half of X X^T, by tiles of 192, 173.
template <typename T, int END, int RN, int CN, int WR, int WC, int SLOTS, int EARLY>
__global__ void __launch_bounds__(WR* WC* kWave) pair_large_kernel(PairTask p) {
  using K = PairKernel<RN, CN, WR, WC, SLOTS>;
  constexpr bool kHalf = END == kGram || END == kPoly;
  constexpr int kAhead = 2, kRingOfA = RN % 4 == 0 ? 4 : 3, kMeet = RN - kAhead, kFirst = kAhead * EARLY, kLate = (K::kLoads - kFirst + kMeet - 1) / kMeet;
  static_assert(RN % kRingOfA == 0 && kFirst <= K::kLoads, "fragments and loads divide evenly");
  __shared__ __align__(1024) char lds[K::kRing];
  const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wr = wave / WC, wc = wave % WC, i = lane % 16;
  const Work w = work_of<K, kHalf>(p);
  Operands<K> of(p, w, lane, wave, lds);
  const uint32_t at_a = (wr * RN * 16 + i) * 128 + (lane / 16 ^ (i >> 1 & 7u)) * 16;
  const uint32_t at_b = (K::kRows + wc * CN * 16 + i) * 128 + (lane / 16 ^ (i >> 1 & 7u)) * 16;
  v8h a[kRingOfA][2], b[2][CN][2];
  auto read_a = [&](int g, uint32_t slot) {
    a[g % kRingOfA][0] = *reinterpret_cast<const v8h*>(lds + slot + at_a + g % RN * 2048);
    a[g % kRingOfA][1] = *reinterpret_cast<const v8h*>(lds + slot + (at_a ^ 64u) + g % RN * 2048);
  };
  auto read_b = [&](int set, int k, uint32_t slot) {
    b[set][k][0] = *reinterpret_cast<const v8h*>(lds + slot + at_b + k * 2048);
    b[set][k][1] = *reinterpret_cast<const v8h*>(lds + slot + (at_b ^ 64u) + k * 2048);
  };
  v4f sum[RN][CN];
#pragma unroll
  for (int k = 0; k < RN; ++k)
#pragma unroll
    for (int n = 0; n < CN; ++n) sum[k][n] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < SLOTS - 1; ++k) {
#pragma unroll
    for (int j = 0; j < K::kLoads; ++j) of.load(j, k * K::kStageBytes);
    of.next();
  }
#pragma unroll
  for (int j = 0; j < kFirst; ++j) of.load(j, (SLOTS - 1) * K::kStageBytes);
  wait_and_meet<(SLOTS - 2) * K::kLoads + kFirst>();
#pragma unroll
  for (int k = 0; k < CN; ++k) read_b(0, k, 0);
#pragma unroll
  for (int k = 0; k < kAhead; ++k) read_a(k, 0);
  uint32_t here = 0;
  auto stage = [&](int set) {
    const uint32_t next = here + K::kStageBytes == K::kRing ? 0u : here + K::kStageBytes, before = here == 0u ? K::kRing - K::kStageBytes : here - K::kStageBytes;
#pragma unroll
    for (int g = 0; g < kMeet; ++g) {
      read_a(g + kAhead, here);
#pragma unroll
      for (int j = kFirst + g * kLate; j < kFirst + (g + 1) * kLate && j < K::kLoads; ++j) of.load(j, before);
      multiply<CN>(sum[g], a[g % kRingOfA], b[set]);
    }
    of.next();
    wait_and_meet<(SLOTS - 2) * K::kLoads>();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = kMeet; g < RN; ++g) {
      read_a(g + kAhead, next);
#pragma unroll
      for (int k = (g - kMeet) * CN / kAhead; k < (g - kMeet + 1) * CN / kAhead; ++k) read_b(1 - set, k, next);
#pragma unroll
      for (int j = (g - kMeet) * EARLY; j < (g - kMeet + 1) * EARLY; ++j) of.load(j, here);
      multiply<CN>(sum[g], a[g % kRingOfA], b[set]);
    }
    here = next;
  };
  uint32_t k = 0;
  for (; k + 2 <= w.stages; k += 2) {
    stage(0);
    stage(1);
  }
  if (k < w.stages) stage(0);
  wait_and_meet<0>();
  finish_tile<T, END, K, RN, CN, WC>(p, w, sum, lds, lane, wave);
}

// The tiles that there are: how many run at a time, what one takes for a stage while as many do, and while no CU has two of them, and what it takes
// besides (us; from products of 64 to 4096 rows, 64 to 4096 deep).
struct Shape {
  uint32_t side, slots;
  double stage, alone, rest;
};
constexpr uint32_t kCus = 256;
constexpr Shape kShapes[] = {{256, 256, 2.0, 2.0, 10.}, {192, 256, 1.25, 1.25, 9.}, {128, 256, 0.55, 0.55, 8.}, {64, 512, 0.34, 0.25, 4.}, {128, 512, 1.1, 0.8, 8.}};

// How a product is made: whatever tiles, and pieces of the tiles that would have the chip to themselves at the end, an estimate of the time says.  (Four
// steps' products of one size with one kind of tile, us: 4096 x 4096 with 256, 192, 128 and 64: 3890, 3500, 4290, 4790, and 3270 by the estimate; 256 x 4096: 1330,
// 830, 490, 240, the last in eight pieces 140.)
struct Plan {
  int shape;
  uint32_t full, rest, splits;  // tiles made whole; others, each by so many workgroups
};
Plan plan_of(bool half, uint32_t rows, uint32_t cols, uint32_t planes, uint32_t stages) {
  Plan best{};
  double least = 1e30;
  int k = 0;
  for (const Shape& s : kShapes) {
    const uint32_t tiles = tiles_of(half, (rows + s.side - 1) / s.side, (cols + s.side - 1) / s.side) * planes;
    // `count` workgroups, each of so many stages
    auto time = [&](uint32_t count, double deep) {
      const uint32_t turns = count / s.slots, left = count - turns * s.slots;
      return turns * (deep * s.stage + s.rest) + (left == 0 ? 0. : deep * (left > kCus ? s.stage : s.alone) + s.rest);
    };
    auto consider = [&](uint32_t full, uint32_t splits, double t) {
      if (t < least) {
        least = t;
        best = Plan{k, full, tiles - full, splits};
      }
    };
    consider(tiles, 1, time(tiles, stages));
    const uint32_t full = tiles / s.slots * s.slots, rest = tiles - full;
    for (uint32_t n = 2; n <= 16 && rest > 0 && stages / n >= 4; ++n)  // (a launch that joins them, and their sums out and in)
      consider(full, n, time(full, stages) + time(rest * n, (double)stages / n) + 5. + rest * n * (s.side * s.side * 8.) / 3e6);
    ++k;
  }
  return best;
}
size_t part_bytes(const Plan& plan) {
  const uint64_t side = kShapes[plan.shape].side;
  return plan.splits > 1 ? plan.rest * (uint64_t)plan.splits * side * side * sizeof(float) : 0;
}

template <typename T, int END>
void product(PairTask p, hipStream_t s) {
  const Plan plan = plan_of(END == kGram || END == kPoly, p.rows, p.cols, p.planes, p.stages);
  p.full = plan.full;
  p.splits = plan.splits;
  auto launch = [&](auto kernel, auto join, uint32_t threads, uint32_t halves) {
    kernel<<<dim3(plan.full + plan.rest * plan.splits), threads, 0, s>>>(p);
    if (plan.rest > 0) join<<<dim3(plan.rest, halves), threads, 0, s>>>(p);
  };
  switch (plan.shape) {
    case 0: launch(pair_large_kernel<T, END, 8, 4, 2, 4, 2, 2>, pair_join_kernel<T, END, 8, 4, 2, 4>, 512, 4); break;
    case 1: launch(pair_large_kernel<T, END, 6, 3, 2, 4, 3, 1>, pair_join_kernel<T, END, 6, 3, 2, 4>, 512, 3); break;
    case 2: launch(pair_kernel<T, END, 4, 2, 2, 4, 4>, pair_join_kernel<T, END, 4, 2, 2, 4>, 512, 2); break;
    case 3: launch(pair_kernel<T, END, 2, 2, 2, 2, 4>, pair_join_kernel<T, END, 2, 2, 2, 2>, 256, 1); break;
    default: launch(pair_kernel<T, END, 4, 4, 2, 2, 2>, pair_join_kernel<T, END, 4, 4, 2, 2>, 256, 2); break;
  }
}

// ---- Small matrices: a workgroup each, everything in one launch; and few rows of longer ones, a strip of columns for each workgroup and a launch a step.
//
// A wavefront holds CT tiles of 16 columns of X, all NT of their tiles of rows, as its matrix instructions leave them: four consecutive rows of a column a
// lane.  P X takes them from there: which of P's columns meets which of X's rows in a lane's eight is free as long as both sides agree, so a lane's
// two fours of rows are its eight, and P's are read from LDS in that order.  Only X X^T wants rows of X, through LDS, where a word is a pair.
constexpr int kSmallWaves = 8, kSmallSteps = 64;

// Eight pairs, or four and four, as fragments.
__device__ __forceinline__ void fragments_of(const uint32_t* first, const uint32_t* second, v8h& high, v8h& low) {
  typedef uint32_t four __attribute__((ext_vector_type(4)));
  const four a = *reinterpret_cast<const four*>(first), b = *reinterpret_cast<const four*>(second);
  four h, l;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    h[k] = __builtin_amdgcn_perm(a[2 * k + 1], a[2 * k], 0x05040100u);
    l[k] = __builtin_amdgcn_perm(a[2 * k + 1], a[2 * k], 0x07060302u);
    h[k + 2] = __builtin_amdgcn_perm(b[2 * k + 1], b[2 * k], 0x05040100u);
    l[k + 2] = __builtin_amdgcn_perm(b[2 * k + 1], b[2 * k], 0x07060302u);
  }
  high = __builtin_bit_cast(v8h, h);
  low = __builtin_bit_cast(v8h, l);
}
__device__ __forceinline__ uint32_t pair_of(float v) {
  f16_t h, l;
  split(v, h, l);
  return (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
}

// What both kernels do; all of a workgroup come to each of these as often as the others.
template <int NT, int CT>
struct Small {
  static_assert(NT % 2 == 0, "a lane's eight are two tiles' fours");
  static constexpr int kRows = NT * 16, kCols = CT * 16 * kSmallWaves, kPitch = kCols + 4, kSquare = kRows + 4, kTiles = NT * (NT + 1) / 2;
  static constexpr int kMine = (kTiles + kSmallWaves - 1) / kSmallWaves;
  typedef uint32_t four __attribute__((ext_vector_type(4)));
  typedef v4f Strip[NT][CT];
  typedef v8h Fragments[NT / 2][CT];
  uint32_t *of_x, *of_p;  // LDS: [kRows][kPitch]; [kRows][kSquare], G, then P
  uint32_t lane, wave, i, g, r_in;

  __device__ __forceinline__ Small(uint32_t* x, uint32_t* p) : of_x(x), of_p(p) {
    lane = threadIdx.x % kWave;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    i = lane % 16;
    g = lane / 16;
    r_in = g * 4;
  }
  __device__ __forceinline__ uint32_t column(int b) const { return wave * CT * 16 + i + b * 16; }

  // n rows and m columns of X, which is what lies there, or, where that is tall, what lies there turned: then a lane's four are side by side.
  template <typename T>
  __device__ __forceinline__ void load(const T* from, bool tall, uint64_t ld, uint32_t n, uint32_t m, Strip& x) const {
    if (tall) {
#pragma unroll
      for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int b = 0; b < CT; ++b) {
          const uint32_t r = r_in + a * 16, c = min(column(b), m - 1);  // (past the end: the last one, which is not used)
          float v[4] = {0.f, 0.f, 0.f, 0.f};
          if (r < n) load_n_within<T, 4>(from + c * ld + r, n - r, 0.f, v);
#pragma unroll
          for (int k = 0; k < 4; ++k) x[a][b][k] = v[k];
          if (b == CT - 1) __builtin_amdgcn_sched_barrier(0);
        }
      return;
    }
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int b = 0; b < CT; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[a][b][k] = (float)from[min(r_in + a * 16 + k, n - 1) * ld + min(column(b), m - 1)];
          if (b == CT - 1 && k == 3) __builtin_amdgcn_sched_barrier(0);
        }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* to, bool tall, uint64_t ld, uint32_t n, uint32_t m, const Strip& x) const {
    // (a barrier behind each tile: so many addresses at once leave no registers)
    if (tall) {
#pragma unroll
      for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int b = 0; b < CT; ++b) {
          const uint32_t r = r_in + a * 16, c = column(b);
          const float v[4] = {x[a][b][0], x[a][b][1], x[a][b][2], x[a][b][3]};
          if (r < n && c < m) store_n_within<T, 4>(to + c * ld + r, n - r, v);
          __builtin_amdgcn_sched_barrier(0);
        }
      return;
    }
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int b = 0; b < CT; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t r = r_in + a * 16 + k, c = column(b);
          if (r < n && c < m) to[r * ld + c] = (T)x[a][b][k];
          if (k == 3) __builtin_amdgcn_sched_barrier(0);
        }
  }
  __device__ __forceinline__ void scale(double inv, uint32_t n, uint32_t m, Strip& x) const {
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int b = 0; b < CT; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[a][b][k] = r_in + a * 16 + k < n && column(b) < m ? (float)((double)x[a][b][k] * inv) : 0.f;
  }

  // X as fragments, and as pairs in LDS.
  template <bool FRAGMENTS, bool LDS>
  __device__ __forceinline__ void divide(const Strip& x, Fragments& high, Fragments& low) const {
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int b = 0; b < CT; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f16_t h, l;
          split(x[a][b][k], h, l);
          if (FRAGMENTS) {
            high[a / 2][b][a % 2 * 4 + k] = h;
            low[a / 2][b][a % 2 * 4 + k] = l;
          }
          if (LDS) of_x[(a * 16 + r_in + k) * kPitch + column(b)] = (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
        }
  }

  // The tile of a number: rows first, c <= r.
  static __device__ __forceinline__ Place place(uint32_t number) {
    uint32_t row = 0;
    while (number > row) number -= ++row;
    return Place{row, number};
  }
  __device__ __forceinline__ void put(const Place& at, const four& pair) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) of_p[(at.r * 16 + r_in + k) * kSquare + at.c * 16 + i] = pair[k];
    if (at.r != at.c) *reinterpret_cast<four*>(of_p + (at.c * 16 + i) * kSquare + at.r * 16 + r_in) = pair;
  }
  // A tile of X X^T times kOfX^2, of what is in LDS.
  __device__ __forceinline__ v4f gram(const Place& at) const {
    v4f main = {0.f, 0.f, 0.f, 0.f}, cross = {0.f, 0.f, 0.f, 0.f};
    const uint32_t *ra = of_x + (at.r * 16 + i) * kPitch + g * 8, *rb = of_x + (at.c * 16 + i) * kPitch + g * 8;
#pragma unroll 2
    for (uint32_t k = 0; k < kCols; k += 32) {
      v8h ah, al, bh, bl;
      fragments_of(ra + k, ra + k + 4, ah, al);
      fragments_of(rb + k, rb + k + 4, bh, bl);
      cross = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bl, cross, 0, 0, 0);
      main = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh, main, 0, 0, 0);
      cross = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, bh, cross, 0, 0, 0);
    }
    return main + cross;
  }
  static __device__ __forceinline__ four pairs_of_gram(const v4f& sum) {
    four pair;
#pragma unroll
    for (int k = 0; k < 4; ++k) pair[k] = pair_of(sum[k] * (kOfGram / (kOfX * kOfX)));
    return pair;
  }

  // P, in the place of G.
  __device__ __forceinline__ void polynomial(float plus, float times, float square) const {
    four made[kMine];
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const uint32_t t = wave + n * kSmallWaves;
      if (t >= kTiles) continue;
      const Place at = place(t);
      v4f all = {0.f, 0.f, 0.f, 0.f};
      const uint32_t *ra = of_p + (at.r * 16 + i) * kSquare + g * 8, *rb = of_p + (at.c * 16 + i) * kSquare + g * 8;
#pragma unroll
      for (uint32_t k = 0; k < kRows; k += 32) {
        v8h ah, al, bh, bl;
        fragments_of(ra + k, ra + k + 4, ah, al);
        fragments_of(rb + k, rb + k + 4, bh, bl);
        all = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bl, all, 0, 0, 0);
        all = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, bh, all, 0, 0, 0);
        all = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh, all, 0, 0, 0);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t word = of_p[(at.r * 16 + r_in + k) * kSquare + at.c * 16 + i];
        const float gram = ((float)__builtin_bit_cast(f16_t, (uint16_t)word) + (float)__builtin_bit_cast(f16_t, (uint16_t)(word >> 16))) * (1.f / kOfGram);
        made[n][k] = pair_of((times * gram + square * (all[k] * (1.f / (kOfGram * kOfGram))) + (at.r == at.c && r_in + k == i ? plus : 0.f)) * kOfPoly);
      }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const uint32_t t = wave + n * kSmallWaves;
      if (t < kTiles) put(place(t), made[n]);
    }
    __syncthreads();
  }

  // P X times unit, a power of two, and then times scale, in the place of X.  (One product for both would be a subnormal number of few bits for scales that
  // results with it are not.)
  __device__ __forceinline__ void apply(const Fragments& high, const Fragments& low, float unit, float scale, Strip& x) const {
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      v4f all[CT] = {};
      const uint32_t* row = of_p + (a * 16 + i) * kSquare + g * 4;
#pragma unroll
      for (int s = 0; s < NT / 2; ++s) {
        v8h ph, pl;
        fragments_of(row + s * 32, row + s * 32 + 16, ph, pl);
#pragma unroll
        for (int b = 0; b < CT; ++b) all[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, low[s][b], all[b], 0, 0, 0);
#pragma unroll
        for (int b = 0; b < CT; ++b) all[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, high[s][b], all[b], 0, 0, 0);
#pragma unroll
        for (int b = 0; b < CT; ++b) all[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, high[s][b], all[b], 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < CT; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[a][b][k] = all[b][k] * unit * scale;
    }
  }
};

template <typename F>
__device__ __forceinline__ void with_type(tng_type type, F f) {
  switch (type) {
    case TNG_TYPE_F32: f(float{}); break;
    case TNG_TYPE_BF16: f(bf16_t{}); break;
    default: f(f16_t{}); break;
  }
}

struct SmallTask {
  uint32_t n, m, steps;
  bool tall;
  View x, y;
  tng_type of_x, of_y;
  float eps, scale;
  float abc[3 * kSmallSteps];
};

// 16 x 64 x 256 in five steps: 28 us, by the latencies of four meetings a step; three launches a step were 80.
template <int NT, int CT>
__global__ void __launch_bounds__(kSmallWaves* kWave) small_kernel(SmallTask p) {
  using K = Small<NT, CT>;
  __shared__ __align__(16) uint32_t of_x[K::kRows * K::kPitch];
  __shared__ __align__(16) uint32_t of_p[K::kRows * K::kSquare];
  __shared__ double of_wave[kSmallWaves];
  const K all(of_x, of_p);
  const uint32_t m = blockIdx.x;
  typename K::Strip x;
  with_type(p.of_x, [&](auto of) {
    using T = decltype(of);
    all.load(static_cast<const T*>(p.x.p) + m * p.x.pitch, p.tall, p.x.ld, p.n, p.m, x);
  });
  double sum = 0.;
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int b = 0; b < CT; ++b)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (all.r_in + a * 16 + k < p.n && all.column(b) < p.m) sum += (double)x[a][b][k] * (double)x[a][b][k];
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  if (all.lane == 0) of_wave[all.wave] = sum;
  __syncthreads();
  sum = 0.;
  for (int k = 0; k < kSmallWaves; ++k) sum += of_wave[k];
  all.scale(inverse_of(sum, p.eps), p.n, p.m, x);
  typename K::Fragments high, low;
  for (uint32_t step = 0; step < p.steps; ++step) {
    all.template divide<true, true>(x, high, low);
    __syncthreads();
#pragma unroll 1
    for (uint32_t t = all.wave; t < K::kTiles; t += kSmallWaves) {
      const Place at = K::place(t);
      all.put(at, K::pairs_of_gram(all.gram(at)));
    }
    __syncthreads();
    all.polynomial(p.abc[3 * step], p.abc[3 * step + 1], p.abc[3 * step + 2]);
    const bool last = step + 1 == p.steps;
    all.apply(high, low, last ? 1.f / (kOfPoly * kOfX) : kOfX / (kOfPoly * kOfX), last ? p.scale : 1.f, x);
  }
  with_type(p.of_y, [&](auto of) {
    using T = decltype(of);
    all.store(static_cast<T*>(p.y.p) + m * p.y.pitch, p.tall, p.y.ld, p.n, p.m, x);
  });
}

struct StripTask {
  uint32_t n, m, step, steps;  // launches 0 .. steps
  bool tall;
  View x, y;
  tng_type of_x, of_y;
  float eps, scale;
  float plus, times, square;  // of step - 1
  const double* part;         // squares: [matrix][parts]
  uint32_t parts;
  float* state;               // [matrix][strip][tile of rows][tile of columns][thread][4]: X, from step 1 on
  const float* sums;          // [matrix][strip][tile of X X^T][lane][4], from the launch before
  float* next;                // the same for the next one
};

// A strip of columns in one step: X X^T from what all strips found of it, P, by every workgroup for itself, P X, and this strip's part of the next X X^T.  Latencies
// bound it: 64 x 1024 in five steps is seven launches of 5 to 7 us, where tiles take three a step and more.
template <int NT, int CT>
__global__ void __launch_bounds__(kSmallWaves* kWave) strip_kernel(StripTask p) {
  using K = Small<NT, CT>;
  __shared__ __align__(16) uint32_t of_x[K::kRows * K::kPitch];
  __shared__ __align__(16) uint32_t of_p[K::kRows * K::kSquare];
  const K all(of_x, of_p);
  const uint32_t m = blockIdx.y, strip = blockIdx.x, strips = gridDim.x;
  const uint32_t c0 = strip * K::kCols, left = p.m - c0;
  typename K::Strip x;
  float* state = p.state + ((uint64_t)m * strips + strip) * (K::kRows * K::kCols) + threadIdx.x * 4;
  if (p.step <= 1) {
    with_type(p.of_x, [&](auto of) {
      using T = decltype(of);
      all.load(static_cast<const T*>(p.x.p) + m * p.x.pitch + c0 * (p.tall ? p.x.ld : 1), p.tall, p.x.ld, p.n, left, x);
    });
    all.scale(inverse_of(sum_of_parts(p.part + (uint64_t)m * p.parts, p.parts, all.lane), p.eps), p.n, left, x);
  } else {
#pragma unroll
    for (int k = 0; k < NT * CT; ++k) x[k / CT][k % CT] = *reinterpret_cast<const v4f*>(state + k * (kSmallWaves * kWave * 4));
  }
  typename K::Fragments high, low;
  if (p.step > 0) {
    const float* sums = p.sums + (uint64_t)m * strips * (K::kTiles * 256) + all.lane * 4;
#pragma unroll 1
    for (uint32_t t = all.wave; t < K::kTiles; t += kSmallWaves) {
      v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (uint32_t k = 0; k < strips; ++k) sum += *reinterpret_cast<const v4f*>(sums + ((uint64_t)k * K::kTiles + t) * 256);
      all.put(K::place(t), K::pairs_of_gram(sum));
    }
    all.template divide<true, false>(x, high, low);
    __syncthreads();
    all.polynomial(p.plus, p.times, p.square);
    const bool last = p.step == p.steps;
    all.apply(high, low, last ? 1.f / (kOfPoly * kOfX) : kOfX / (kOfPoly * kOfX), last ? p.scale : 1.f, x);
    if (last) {
      with_type(p.of_y, [&](auto of) {
        using T = decltype(of);
        all.store(static_cast<T*>(p.y.p) + m * p.y.pitch + c0 * (p.tall ? p.y.ld : 1), p.tall, p.y.ld, p.n, left, x);
      });
      return;
    }
#pragma unroll
    for (int k = 0; k < NT * CT; ++k) *reinterpret_cast<v4f*>(state + k * (kSmallWaves * kWave * 4)) = x[k / CT][k % CT];
  }
  all.template divide<false, true>(x, high, low);
  __syncthreads();
  float* next = p.next + ((uint64_t)m * strips + strip) * (K::kTiles * 256) + all.lane * 4;
#pragma unroll 1
  for (uint32_t t = all.wave; t < K::kTiles; t += kSmallWaves) *reinterpret_cast<v4f*>(next + t * 256) = all.gram(K::place(t));
}

// As many columns as LDS holds beside the rows, in turns of 128.
inline bool is_small(uint64_t n, uint64_t m) { return m <= (n <= 32 ? 1024u : n <= 64 ? 512u : n <= 96 ? 256u : n <= 128 ? 128u : 0u); }

hipError_t launch_small(const SmallTask& p, uint32_t workers, hipStream_t s) {
  auto launch = [&](auto rows, auto cols) { small_kernel<rows, cols><<<dim3(workers), kSmallWaves * kWave, 0, s>>>(p); };
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  constexpr std::integral_constant<int, 4> four;
  constexpr std::integral_constant<int, 8> eight;
  constexpr std::integral_constant<int, 6> six;
  auto up_to_256 = [&](auto rows) { p.m <= 128 ? launch(rows, one) : launch(rows, two); };
  auto up_to_512 = [&](auto rows) { p.m <= 256 ? up_to_256(rows) : launch(rows, four); };
  if (p.n <= 32)
    p.m <= 512 ? up_to_512(two) : launch(two, eight);
  else if (p.n <= 64)
    up_to_512(four);
  else if (p.n <= 96)
    up_to_256(six);
  else
    launch(eight, one);
  return hipGetLastError();
}

// Strips of this many columns, or 0: not by strips.  Every strip reads what all of them found of X X^T, so there are no more than sixteen.  (Five
// steps, us, and by tiles: 64 x 1024 46 and 104, 32 x 4096 37 and 108, 64 x 8192 85 and 127, 100 x 64 x 1024 144 and 190, 100 x 64 x 8000 740 and 1055, with up to
// 32 strips 77 and 1128 of the last 85 and 740; 96 x 1000 69 and 100, 64 x 96 x 1000 204 and 188, so not where the chip is full anyway.)
constexpr uint32_t kMostStrips = 16;
uint32_t strip_of(const Extent& e) {
  const uint64_t n = std::min(e.rows, e.cols), m = std::max(e.rows, e.cols);
  const uint32_t most = n <= 64 ? 512 : n <= 96 ? 256 : 0;  // (LDS has room for no more)
  for (uint32_t cols = 128; cols <= most; cols *= 2) {
    const uint64_t strips = (m + cols - 1) / cols;
    if (strips <= kMostStrips) return n <= 64 || e.workers * strips <= kCus ? cols : 0;
  }
  return 0;
}

struct Strips {
  uint64_t n, m;
  uint32_t cols, count, parts;
  double* part;
  float *state, *sums[2];
  uint64_t bytes;
};
uint32_t squares_parts(const Extent& e) {  // (four pieces of a row for each wavefront)
  const uint64_t pieces = e.rows * ((e.cols + kWave * 8 - 1) / (kWave * 8));
  return (uint32_t)std::min<uint64_t>(std::max<uint64_t>(1, 1024 / e.workers), (pieces + 15) / 16);
}
Strips strips_of(const Extent& e, char* scratch) {
  Strips l{};
  l.n = std::min(e.rows, e.cols);
  l.m = std::max(e.rows, e.cols);
  l.cols = strip_of(e);
  l.count = (uint32_t)((l.m + l.cols - 1) / l.cols);
  l.parts = squares_parts(e);
  auto take = [&](uint64_t bytes) {
    char* here = scratch + l.bytes;
    l.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  const uint64_t tiles = (l.n + 31) / 32 * 2, all = e.workers * (uint64_t)l.count;
  l.part = reinterpret_cast<double*>(take(e.workers * (uint64_t)l.parts * sizeof(double)));
  l.state = reinterpret_cast<float*>(take(all * tiles * 16 * l.cols * sizeof(float)));
  for (float*& sums : l.sums) sums = reinterpret_cast<float*>(take(all * (tiles * (tiles + 1) / 2 * 256) * sizeof(float)));
  return l;
}
void launch_strip(const StripTask& p, const Strips& l, uint32_t workers, hipStream_t s) {
  auto launch = [&](auto rows, auto cols) { strip_kernel<rows, cols><<<dim3(l.count, workers), kSmallWaves * kWave, 0, s>>>(p); };
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  constexpr std::integral_constant<int, 4> four;
  constexpr std::integral_constant<int, 6> six;
  auto of_rows = [&](auto rows) { l.cols == 128 ? launch(rows, one) : l.cols == 256 ? launch(rows, two) : launch(rows, four); };
  if (l.n <= 32)
    of_rows(two);
  else if (l.n <= 64)
    of_rows(four);
  else
    l.cols == 128 ? launch(six, one) : launch(six, two);
}

struct Layout {
  uint64_t n, m;
  bool tall;
  uint32_t parts;
  Pairs x_by_n, x_by_m[2], gram, poly;
  double* part;
  float* sums;  // of tiles that are made in pieces
  uint64_t bytes;
};

Layout layout_of(const Extent& e, char* scratch) {
  Layout l{};
  l.tall = e.rows > e.cols;
  l.n = std::min(e.rows, e.cols);
  l.m = std::max(e.rows, e.cols);
  l.parts = squares_parts(e);
  auto take = [&](uint64_t bytes) {
    char* here = scratch + l.bytes;
    l.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  auto pairs = [&](uint64_t rows, uint64_t cols) {
    const uint64_t ld = pair_row(cols);
    return Pairs{take(e.workers * rows * ld), ld, rows * ld};
  };
  l.part = reinterpret_cast<double*>(take(e.workers * (uint64_t)l.parts * sizeof(double)));
  l.x_by_n = pairs(l.n, l.m);
  for (Pairs& x : l.x_by_m) x = pairs(l.m, l.n);
  l.gram = pairs(l.n, l.n);
  l.poly = pairs(l.n, l.n);
  const uint32_t n = (uint32_t)l.n, m = (uint32_t)l.m, n_stages = (n + kBlockCols - 1) / kBlockCols, m_stages = (m + kBlockCols - 1) / kBlockCols;
  l.sums = reinterpret_cast<float*>(take(std::max({part_bytes(plan_of(true, n, n, e.workers, m_stages)), part_bytes(plan_of(true, n, n, e.workers, n_stages)),
                                                   part_bytes(plan_of(false, n, m, e.workers, n_stages)), part_bytes(plan_of(false, m, n, e.workers, n_stages))})));
  return l;
}

template <typename T>
void start(const StartTask& p, uint32_t workers, hipStream_t s) {
  squares_kernel<T><<<dim3(p.parts, workers), kBlock, 0, s>>>(p);
  if (p.x_by_n.p == nullptr) return;
  start_kernel<T><<<dim3((uint32_t)((p.cols + kTurn - 1) / kTurn), (uint32_t)((p.rows + kTurn - 1) / kTurn), workers), kBlock, 0, s>>>(p);
}

}  // namespace

// The largest |s p(s^2)| and |p(s^2)| of s in 0 .. top, p(t) = a + b t + c t^2: at the ends, or where a derivative is 0.
static void reach(const float* abc, double top, double* of_x, double* of_p) {
  const double a = abc[0], b = abc[1], c = abc[2], end = top * top;
  auto p = [&](double t) { return std::fabs(a + t * (b + t * c)); };
  *of_p = std::max(p(0.), p(end));
  *of_x = std::sqrt(end) * p(end);
  auto at = [&](double t) {
    if (!(t > 0. && t < end)) return;
    *of_p = std::max(*of_p, p(t));
    *of_x = std::max(*of_x, std::sqrt(t) * p(t));
  };
  at(-b / (2. * c));
  const double root = 9. * b * b - 20. * a * c;  // of a + 3 b t + 5 c t^2
  if (root >= 0.) {
    at((-3. * b + std::sqrt(root)) / (10. * c));
    at((-3. * b - std::sqrt(root)) / (10. * c));
  }
  at(-a / (3. * b));  // (c = 0)
}

bool orthogonal_in_range(const float* coefficients, uint32_t steps) {
  double top = 1.;
  for (uint32_t k = 0; k < steps; ++k) {
    double of_x, of_p;
    reach(coefficients + 3 * k, top, &of_x, &of_p);
    if (!(of_p < 7.9)) return false;  // (of pairs up to 8 2^13, a little less than 2^16)
    top = of_x * 1.001;               // what rounding may add
    if (!(top < 1.98)) return false;
  }
  return true;
}

size_t orthogonal_bytes(const Extent& e) {
  const uint64_t n = std::min(e.rows, e.cols), m = std::max(e.rows, e.cols);
  return is_small(n, m) ? 0 : strip_of(e) != 0 ? strips_of(e, nullptr).bytes : layout_of(e, nullptr).bytes;
}

hipError_t launch_orthogonalize(tng_type of_x, tng_type of_y, const Extent& e, const View& x, const float* coefficients, uint32_t steps, float eps, float scale,
                                const View& y, char* scratch, hipStream_t s) {
  if (is_small(std::min(e.rows, e.cols), std::max(e.rows, e.cols))) {
    SmallTask small{(uint32_t)std::min(e.rows, e.cols), (uint32_t)std::max(e.rows, e.cols), steps, e.rows > e.cols, x, y, of_x, of_y, eps, scale, {}};
    std::copy(coefficients, coefficients + 3 * steps, small.abc);
    return launch_small(small, e.workers, s);
  }
  auto begin = [&](const StartTask& first) {
    switch (of_x) {
      case TNG_TYPE_F32: start<float>(first, e.workers, s); break;
      case TNG_TYPE_BF16: start<bf16_t>(first, e.workers, s); break;
      default: start<f16_t>(first, e.workers, s); break;
    }
  };
  if (strip_of(e) != 0) {
    const Strips l = strips_of(e, scratch);
    begin(StartTask{e.rows, e.cols, x, l.part, l.parts, eps, false, {}, {}});
    StripTask p{(uint32_t)l.n, (uint32_t)l.m, 0, steps, e.rows > e.cols, x, y, of_x, of_y, eps, scale, 0.f, 0.f, 0.f, l.part, l.parts, l.state, nullptr, nullptr};
    for (; p.step <= steps; ++p.step) {
      if (p.step > 0) {
        p.plus = coefficients[3 * p.step - 3];
        p.times = coefficients[3 * p.step - 2];
        p.square = coefficients[3 * p.step - 1];
      }
      p.sums = l.sums[(p.step + 1) % 2];
      p.next = l.sums[p.step % 2];
      launch_strip(p, l, e.workers, s);
    }
    return hipGetLastError();
  }
  const Layout l = layout_of(e, scratch);
  begin(StartTask{e.rows, e.cols, x, l.part, l.parts, eps, l.tall, l.x_by_n, l.x_by_m[0]});
  const uint32_t n = (uint32_t)l.n, m = (uint32_t)l.m, n_stages = (n + kBlockCols - 1) / kBlockCols, m_stages = (m + kBlockCols - 1) / kBlockCols;
  for (uint32_t k = 0; k < steps; ++k) {
    const Pairs &now = l.x_by_m[k % 2], &then = l.x_by_m[1 - k % 2];
    PairTask gram{};
    gram.rows = gram.cols = n;
    gram.stages = m_stages;
    gram.planes = e.workers;
    gram.a = gram.b = l.x_by_n;
    gram.by_r = gram.by_c = l.gram;
    gram.part = l.sums;
    product<float, kGram>(gram, s);
    PairTask poly = gram;
    poly.stages = n_stages;
    poly.a = poly.b = poly.gram = l.gram;
    poly.plus = coefficients[3 * k];
    poly.times = coefficients[3 * k + 1];
    poly.square = coefficients[3 * k + 2];
    poly.by_r = poly.by_c = l.poly;
    product<float, kPoly>(poly, s);
    PairTask apply{};
    apply.planes = e.workers;
    apply.part = l.sums;
    apply.stages = n_stages;
    const bool last = k + 1 == steps;
    // (the last one's results lie along r where y's rows do)
    const bool turned = last && !l.tall;
    apply.rows = turned ? m : n;
    apply.cols = turned ? n : m;
    apply.a = turned ? now : l.poly;
    apply.b = turned ? l.poly : now;
    apply.by_r = l.x_by_n;
    apply.by_c = then;
    apply.y = y;
    apply.scale = scale;
    if (!last) {
      product<float, kApply>(apply, s);
    } else {
      switch (of_y) {
        case TNG_TYPE_F32: product<float, kLast>(apply, s); break;
        case TNG_TYPE_BF16: product<bf16_t, kLast>(apply, s); break;
        default: product<f16_t, kLast>(apply, s); break;
      }
    }
  }
  return hipGetLastError();
}

}  // namespace tng
