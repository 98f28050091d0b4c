// Matrices orthogonalised by Newton-Schulz products on the matrix units (gfx950).
//
//   X = x / (||x|| + eps);  a step: G = X X^T,  E = b G + c G G,  X' = a X + E X
//
// with X lying so that it has no more rows n than columns m.  G and E are symmetric: only half of them is computed.
//
// X is held in binary32 from step to step.  The operands of products are pairs of binary16, v = high + low with low = v - high rounded: 22 bits of v and more, as
// long as low is no subnormal number.  So every row of an operand is held times a power of two of its own, which goes by the row's norm and is taken from the
// sums again: what is lost of a row is measured by that row, not by the largest one, whether rows of X are small or columns (those are the rows of the
// other operand of E X).  A product of pairs is three products, high high + high low + low high (low low is below the last bit), summed in binary32: three
// times the work at sixteen times the rate of binary32, and row by row and column by column as near to binary64 within a factor of four, mostly nearer.  512 x 1024
// with rows spread over 1 to 1e-6, the worst row's error: 8e-8 after one step and 6e-6 after five, where binary32's products have 7e-8 and 9e-6.  (Of one power for
// all rows 7e-5 and 2e-4, and rows of 1e-12 were lost.)  Bits of 16 alone would not do: what rounding takes from a direction of small singular value grows with
// it, by 3.4 a step.
#include "tng_layer_device.hpp"
#include "tng_pair_loads.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace tng {
namespace {

typedef f16_t v2h __attribute__((ext_vector_type(2)));
typedef f16_t v4h __attribute__((ext_vector_type(4)));
typedef f16_t v8h __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));

// The powers of two.  A row of X (or a column) whose norm begins at 2^-p or below stays at 2^(c - p) or below, where 2^c is what the polynomials so far can
// have made of a norm, and below 2, as singular values do.  It is held times 2^held, which leaves no number above 2^15; its row of G, not longer by more than
// the largest singular value, the same; its row of E times 2^(held - u), where u goes by the step's b and c.  p goes up to kMostDown: rows below 2^-60 of
// the matrix lose bits against 2^-99 of it.
constexpr int kMostDown = 60;
__device__ __forceinline__ int held(int p, int c) { return 15 + max(p - c, -1); }
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ float inverse_two(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }
// p of a norm.  (What is not finite, and 0: no matter.)
__device__ __forceinline__ int down_of(float norm) { return min(max(-__builtin_amdgcn_frexp_expf(norm), 0), kMostDown); }

// A matrix of pairs: rows of blocks of 32 columns, 128 bytes each: the high parts, then the low parts.  What lies between the last column and the end of
// its block is 0.
constexpr uint32_t kBlockCols = 32;
constexpr uint64_t kBlockBytes = 128;
inline uint64_t pair_row(uint64_t cols) { return (cols + kBlockCols - 1) / kBlockCols * kBlockBytes; }

struct Pairs {
  char* p;
  uint64_t ld, pitch;  // bytes from row to row, and from matrix to matrix
};
// The same of numbers of 32 bits: 128 bytes hold as many columns.  Of each eight columns the first four lie in the first half of them and the others in the second,
// so that a lane finds its eight where it finds the high and the low parts of a pair's.
using Rows = Pairs;
__host__ __device__ inline uint32_t float_at(uint32_t col) { return col / kBlockCols * (uint32_t)kBlockBytes + col % kBlockCols / 8 * 16 + col / 4 % 2 * 64 + col % 4 * 4; }
__host__ __device__ inline uint64_t pair_at(uint64_t col) { return col / kBlockCols * kBlockBytes + col % kBlockCols * 2; }

// Two numbers, times powers of two, as pairs.  (The difference is exact in binary32.  Binary32 is pinned in between: a product or difference and its rounding as one
// instruction, which the compiler has, takes the time of three.)
__device__ __forceinline__ v2h rounded(float a, float b) { return __builtin_convertvector((v2f{a, b}), v2h); }
__device__ __forceinline__ float rest_of(float v, float up, f16_t high) { return pinned(__builtin_fmaf(v, up, -(float)high)); }
__device__ __forceinline__ void split(float a, float b, float up_a, float up_b, v2h& high, v2h& low) {
  high = rounded(pinned(a * up_a), pinned(b * up_b));
  low = rounded(rest_of(a, up_a, high[0]), rest_of(b, up_b, high[1]));
}
// One, as a word.
__device__ __forceinline__ uint32_t pair_of(float v, float up) {
  const float whole = pinned(v * up);
  return __builtin_bit_cast(uint32_t, rounded(whole, rest_of(v, up, (f16_t)whole)));
}
__device__ __forceinline__ float value_of(uint32_t pair) {
  return (float)__builtin_bit_cast(f16_t, (uint16_t)pair) + (float)__builtin_bit_cast(f16_t, (uint16_t)(pair >> 16));
}

// A step: X' = a X + (b G + c G G) X; and the powers of two that go with it.
struct Step {
  float a, b, c;
  int before, after, poly;  // c of held() at its beginning and at its end, u
};

// ---- ||x||, the norms of rows and columns, and x as pairs both ways round

// Workgroups of a matrix: `strips` of rows by `chunks` of 512 columns; `lanes` of a wavefront share a row.
struct NormsTask {
  uint64_t rows, cols;  // of x as it lies
  View x;
  uint32_t lanes, chunks, strips;
  double *part, *by_row, *by_col;  // squares: [matrix][strip][chunk], [matrix][chunk][row], [matrix][strip][column]
};
constexpr uint32_t kChunk = kWave * 8;

template <int CTRL, int ROWS>
__device__ __forceinline__ double plus_other(double x) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, x);
  const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, ROWS, 0xF, false);
  const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, ROWS, 0xF, false);
  return x + __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
// The sum over a wavefront, in its last lane.
__device__ __forceinline__ double sum_of_wave(double x) {
  x = plus_other<0xB1, 0xF>(x);
  x = plus_other<0x4E, 0xF>(x);
  x = plus_other<0x141, 0xF>(x);
  x = plus_other<0x140, 0xF>(x);
  x = plus_other<0x142, 0xA>(x);
  return plus_other<0x143, 0xC>(x);
}

// Squares are summed in binary64, which holds those of every number, in a fixed order.
template <typename T>
__global__ void __launch_bounds__(kBlock) norms_kernel(NormsTask p) {
  constexpr uint32_t kWaves = kBlock / kWave;
  __shared__ double of_wave[kWaves][kChunk];
  __shared__ double of_all[kWaves];
  const uint32_t m = blockIdx.y, chunk = blockIdx.x % p.chunks, strip = blockIdx.x / p.chunks;
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, each = kWave / p.lanes, sub = lane / p.lanes, in = lane % p.lanes;
  const T* x = static_cast<const T*>(p.x.p) + m * p.x.pitch;
  const uint64_t first = p.rows * strip / p.strips, end = p.rows * (strip + 1) / p.strips, c = (uint64_t)chunk * kChunk + in * 8;
  double* by_row = p.by_row + ((uint64_t)m * p.chunks + chunk) * p.rows;
  double col[8] = {0., 0., 0., 0., 0., 0., 0., 0.};
  constexpr int kMany = 4;  // rows that are on the way together
  for (uint64_t r0 = first + wave * each + sub; r0 - sub < end; r0 += kMany * kWaves * each) {
    float v[kMany][8];
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      const uint64_t r = r0 + k * (kWaves * each);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
      if (r < end && c < p.cols) load_n_within<T, 8>(x + r * p.x.ld + c, p.cols - c, 0.f, v[k]);
    }
    double sum[kMany];
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      sum[k] = 0.;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double x = (double)v[k][i];
        col[i] = __builtin_fma(x, x, col[i]);  // (squares are exact)
        sum[k] = __builtin_fma(x, x, sum[k]);
      }
    }
    if (p.lanes == kWave) {
#pragma unroll
      for (int k = 0; k < kMany; ++k) sum[k] = sum_of_wave(sum[k]);
    } else {
      for (uint32_t off = 1; off < p.lanes; off *= 2)
#pragma unroll
        for (int k = 0; k < kMany; ++k) sum[k] += __shfl_xor(sum[k], (int)off, kWave);
    }
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      const uint64_t r = r0 + k * (kWaves * each);
      if (in == p.lanes - 1 && r < end) by_row[r] = sum[k];
    }
  }
  for (uint32_t off = p.lanes; off < kWave; off *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i) col[i] += __shfl_xor(col[i], (int)off, kWave);
  if (sub == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) of_wave[wave][in * 8 + i] = col[i];
  }
  __syncthreads();
  double all = 0.;
  for (uint32_t k = threadIdx.x; k < p.lanes * 8; k += kBlock) {
    double sum = 0.;
    for (uint32_t w = 0; w < kWaves; ++w) sum += of_wave[w][k];
    if ((uint64_t)chunk * kChunk + k < p.cols) p.by_col[((uint64_t)m * p.strips + strip) * p.cols + (uint64_t)chunk * kChunk + k] = sum;
    all += sum;
  }
  for (int off = 32; off > 0; off >>= 1) all += __shfl_xor(all, off, kWave);
  if (lane == 0) of_all[wave] = all;
  __syncthreads();
  if (threadIdx.x != 0) return;
  all = 0.;
  for (uint32_t w = 0; w < kWaves; ++w) all += of_all[w];
  p.part[(uint64_t)m * (p.chunks * p.strips) + blockIdx.x] = all;
}

__device__ __forceinline__ double sum_of_parts(const double* part, uint32_t parts, uint32_t lane) {
  double sum = 0.;
  for (uint32_t k = lane; k < parts; k += kWave) sum += part[k];
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  return sum;
}
// What x is multiplied by, from its squares.  (A matrix that holds what is not finite is NaN as a whole.)
__device__ __forceinline__ double inverse_of(double squares, float eps) {
  return squares < __builtin_inf() ? 1. / (sqrt(squares) + (double)eps) : __builtin_nan("");
}

// p of 64 rows (or columns), by 256 lanes: a quarter of the sums each.  joined: [4][64].
__device__ __forceinline__ int down_of_sums(const double* sums, uint32_t count, uint64_t n, uint64_t first, double inverse, double (*joined)[kWave], uint32_t t) {
  const uint64_t k = first + t % kWave;
  double sum = 0.;
  if (k < n) {
#pragma unroll 4
    for (uint32_t s = t / kWave; s < count; s += 4) sum += sums[s * n + k];
  }
  joined[t / kWave][t % kWave] = sum;
  __syncthreads();
  sum = 0.;
  for (int s = 0; s < 4; ++s) sum += joined[s][t % kWave];
  return down_of((float)(sqrt(sum) * inverse));
}

struct DownTask {
  uint64_t rows, cols;
  uint32_t chunks, strips;
  const double *part, *by_row, *by_col;
  float eps;
  int32_t *of_row, *of_col;  // p: [matrix][rows, columns, up to a multiple of 64]
};
inline uint64_t downs(uint64_t n) { return (n + kWave - 1) / kWave * kWave; }

// p of every row and column, 64 a workgroup, those of the rows first.
__global__ void __launch_bounds__(kBlock) downs_kernel(DownTask p) {
  __shared__ double joined[4][kWave];
  __shared__ double inverse;
  const uint32_t m = blockIdx.y, of_rows = (uint32_t)((p.rows + kWave - 1) / kWave), parts = p.chunks * p.strips;
  if (threadIdx.x < kWave) {
    const double sum = sum_of_parts(p.part + (uint64_t)m * parts, parts, threadIdx.x);
    if (threadIdx.x == 0) inverse = inverse_of(sum, p.eps);
  }
  __syncthreads();
  const bool rows = blockIdx.x < of_rows;
  const uint64_t n = rows ? p.rows : p.cols, first = (uint64_t)(rows ? blockIdx.x : blockIdx.x - of_rows) * kWave;
  const double* sums = rows ? p.by_row + (uint64_t)m * p.chunks * n : p.by_col + (uint64_t)m * p.strips * n;
  const int down = down_of_sums(sums, rows ? p.chunks : p.strips, n, first, inverse, joined, threadIdx.x);
  if (threadIdx.x < kWave) (rows ? p.of_row : p.of_col)[m * ((n + kWave - 1) / kWave * kWave) + first + threadIdx.x] = down;
}

struct StartTask {
  uint64_t rows, cols;  // of x as it lies
  View x;
  const double* part;  // [matrix][parts]
  uint32_t parts;
  float eps;
  bool tall;  // x has more rows than columns: X is x turned
  const int32_t *of_row, *of_col;
  Pairs x_by_n;    // X
  Rows x_turned;   // X turned, as it is held
};

// 64 x 64 elements of x for a workgroup: X as pairs, and X turned in binary32.
constexpr uint32_t kTurn = 64;

template <typename T>
__global__ void __launch_bounds__(kBlock) start_kernel(StartTask p) {
  __shared__ float tile[kTurn][kTurn + 1];  // [row][column]
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
  const int32_t *of_row = p.of_row + m * ((p.rows + kWave - 1) / kWave * kWave), *of_col = p.of_col + m * ((p.cols + kWave - 1) / kWave * kWave);
  const uint32_t eight = threadIdx.x % 8, line = threadIdx.x / 8;
  auto put = [&](bool turned, uint64_t row, uint64_t col, int down, const float (&v)[8]) {
    const float up = two_to(held(down, 0));
    if (turned) {
      char* to = p.x_turned.p + m * p.x_turned.pitch + row * p.x_turned.ld + float_at((uint32_t)col);
      *reinterpret_cast<v4f*>(to) = v4f{v[0], v[1], v[2], v[3]} * up;
      *reinterpret_cast<v4f*>(to + 64) = v4f{v[4], v[5], v[6], v[7]} * up;
      return;
    }
    v8h high, low;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      v2h h, l;
      split(v[i], v[i + 1], up, up, h, l);
      high[i] = h[0];
      high[i + 1] = h[1];
      low[i] = l[0];
      low[i + 1] = l[1];
    }
    char* to = p.x_by_n.p + m * p.x_by_n.pitch + row * p.x_by_n.ld + pair_at(col);
    *reinterpret_cast<v8h*>(to) = high;
    *reinterpret_cast<v8h*>(to + 64) = low;
  };
#pragma unroll
  for (uint32_t k = 0; k < kTurn; k += kBlock / 8) {
    const uint64_t r = r0 + k + line, c = c0 + eight * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (r < p.rows && c < p.cols) load_n_within<T, 8>(x + r * p.x.ld + c, p.cols - c, 0.f, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = r < p.rows && c + i < p.cols ? (float)((double)v[i] * inv) : 0.f;
      tile[k + line][eight * 8 + i] = v[i];
    }
    if (r < p.rows && c < (p.cols + kBlockCols - 1) / kBlockCols * kBlockCols) put(p.tall, r, c, of_row[r], v);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < kTurn; k += kBlock / 8) {
    const uint64_t c = c0 + k + line, r = r0 + eight * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = tile[eight * 8 + i][k + line];
    if (c < p.cols && r < (p.rows + kBlockCols - 1) / kBlockCols * kBlockCols) put(!p.tall, c, r, of_col[c], v);
  }
}

// ---- products of pairs: result (r, c) is the sum over k of a(r, k) b(c, k)

// What becomes of the sums.
constexpr int kGram = 0, kPoly = 1, kApply = 2, kLast = 3;

struct PairTask {
  uint32_t rows, cols, stages;  // rows of a, of b; blocks of 32 that they are long
  uint32_t planes;
  Pairs a, b;                   // kApply, kLast: b is X turned, as it is held but in binary32: pairs are made of it on the way to the matrix units
  const int32_t *of_r, *of_c;  // p of what r and c count, [matrix][up to a multiple of 64]
  uint64_t pitch_r, pitch_c;
  int before, after, poly;    // c of the step and of the next one, u
  Rows gram;                  // kGram, kPoly: G in binary32, where c is no more than r, as rows of c
  float plus, times, square;  // a, b, c
  Pairs by_r, by_c;           // results as rows of r, and turned, as rows of c (kApply: in x_then)
  Rows x_then;                // kApply: X turned, as it is held, from b, which is X turned before
  bool tall;                  // kLast: y's rows are rows of c
  View y;
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
// tile's beginning and end pass while the other is multiplied: 6 % of 4 x 2053 x 1003, 11 % of 100 x 256 x 256.  (A meeting every other stage, with five in
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

// What two tiles of rows, from r_first on, of a wavefront's results want to know: p of rows of r, and X or G in binary32 where the results are.  (G as pairs would do for
// one of the two rows that want an element of E: of the other one's it may be nothing.)
typedef int32_t v4i __attribute__((ext_vector_type(4)));
template <int CN>
struct Found {
  v4i down_r[2];
  v4f old[2][CN];
};
template <int END, int CN>
__device__ __forceinline__ void find_rows(const PairTask& p, uint32_t plane, bool both, uint32_t r_first, uint32_t c_first, uint32_t lane, Found<CN>& found) {
  // A lane has four results of consecutive r for one c.
  const uint32_t r_in = r_first + lane / 16 * 4, c_in = c_first + lane % 16, end_r = (p.rows + kBlockCols - 1) / kBlockCols * kBlockCols;
#pragma unroll
  for (int a = 0; a < 2; ++a) found.down_r[a] = *reinterpret_cast<const v4i*>(p.of_r + plane * p.pitch_r + min(r_in + a * 16, end_r - 4));
  if (END == kGram) return;
  const Rows& rows = END == kPoly ? p.gram : p.b;
  const char* from = rows.p + plane * rows.pitch;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < CN; ++b) {
      const uint32_t r = r_in + a * 16, c = c_in + b * 16;
      v4f& old = found.old[a][b];
      old = v4f{0.f, 0.f, 0.f, 0.f};
      if (END != kPoly || both) {
        if (c < p.cols && r < end_r) old = *reinterpret_cast<const v4f*>(from + c * rows.ld + float_at(r));
      } else {  // (G where c is more than r)
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n)
          if (r + n < p.rows && c < p.cols) old[n] = *reinterpret_cast<const float*>(from + min(c, r + n) * rows.ld + float_at(max(c, r + n)));
      }
    }
}
// p of a wavefront's c.
template <int CN>
__device__ __forceinline__ void find_columns(const PairTask& p, uint32_t plane, uint32_t c_first, uint32_t lane, int (&down)[CN]) {
#pragma unroll
  for (int b = 0; b < CN; ++b) down[b] = p.of_c[plane * p.pitch_c + min(c_first + lane % 16 + b * 16, p.cols - 1)];
}

// What becomes of the results; turn: the wavefront's place in LDS.  both: results go both ways round.
template <typename T, int END, int CN>
__device__ __forceinline__ void finish_rows(const PairTask& p, uint32_t plane, bool both, uint32_t r_first, uint32_t c_first, const v4f (&sum)[2][CN],
                                            const Found<CN>& found, const int (&down_c)[CN], uint32_t* turn, uint32_t lane) {
  constexpr uint32_t kPitch = turn_pitch(CN);
  const uint32_t i = lane % 16, r_in = r_first + lane / 16 * 4, c_in = c_first + i;
  const uint32_t end_r = (p.rows + kBlockCols - 1) / kBlockCols * kBlockCols, end_c = (p.cols + kBlockCols - 1) / kBlockCols * kBlockCols;
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < CN; ++b) {
      const uint32_t r = r_in + a * 16, c = c_in + b * 16;
      const int held_c = held(down_c[b], p.before);
      const bool in = c < p.cols && r < end_r;
      // What becomes of a sum, and the powers that it is held times as rows of c and of r.
      float v[4], up_c[4], up_r[4];
      const float less_c = two_to(-held_c);
      if (END == kGram || END == kPoly) {
        v4f gram;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int held_r = held(found.down_r[a][n], p.before);
          const float less_r = two_to(-held_r), unit = sum[a][b][n] * less_r * less_c;  // (sums are times both rows' powers)
          if (END == kGram) {
            v[n] = sum[a][b][n];
            gram[n] = unit;
            up_c[n] = less_r;
            up_r[n] = less_c;
          } else {
            v[n] = p.times * found.old[a][b][n] + p.square * unit;
            up_c[n] = two_to(held_c - p.poly);
            up_r[n] = two_to(held_r - p.poly);
          }
        }
        if (END == kGram && in) *reinterpret_cast<v4f*>(p.gram.p + plane * p.gram.pitch + c * p.gram.ld + float_at(r)) = gram;
      } else {
        v4f x;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          v[n] = (p.plus * found.old[a][b][n] + sum[a][b][n] * two_to(p.poly - held(found.down_r[a][n], p.before))) * less_c;
          x[n] = r + n < p.rows ? v[n] : 0.f;  // (columns that there are none of are 0 in operands)
        }
        if (END == kLast) {
#pragma unroll
          for (int n = 0; n < 4; ++n) v[n] *= p.scale;
          if (!p.tall) {
#pragma unroll
            for (int n = 0; n < 4; ++n) turn[(a * 16 + lane / 16 * 4 + n) * kPitch + b * 16 + i] = __float_as_uint(v[n]);
          } else if (r < p.rows && c < p.cols) {
            store_n_within<T, 4>(static_cast<T*>(p.y.p) + plane * p.y.pitch + c * p.y.ld + r, p.rows - r, v);
          }
          continue;
        }
        if (in) *reinterpret_cast<v4f*>(p.x_then.p + plane * p.x_then.pitch + c * p.x_then.ld + float_at(r)) = x * two_to(held(down_c[b], p.after));
#pragma unroll
        for (int n = 0; n < 4; ++n)
          turn[(a * 16 + lane / 16 * 4 + n) * kPitch + b * 16 + i] =
              pair_of(c < p.cols ? x[n] : 0.f, two_to(held(found.down_r[a][n], p.after)));
        continue;
      }
      v4h high, low;
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = r + n < p.rows && c < p.cols ? v[n] : 0.f;
      if (both) {
#pragma unroll
        for (int n = 0; n < 4; ++n) turn[(a * 16 + lane / 16 * 4 + n) * kPitch + b * 16 + i] = pair_of(v[n], up_r[n]);
      }
#pragma unroll
      for (int n = 0; n < 4; n += 2) {
        v2h h, l;
        split(v[n], v[n + 1], up_c[n], up_c[n + 1], h, l);
        high[n] = h[0];
        high[n + 1] = h[1];
        low[n] = l[0];
        low[n + 1] = l[1];
      }
      if (in) {
        char* at = p.by_c.p + plane * p.by_c.pitch + c * p.by_c.ld + pair_at(r);
        *reinterpret_cast<v4h*>(at) = high;
        *reinterpret_cast<v4h*>(at + 64) = low;
      }
    }
  if (END == kLast ? p.tall : !both) return;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wavefront's own: what its lanes have written is there)
  constexpr uint32_t kEights = CN * 2;                // of a row
  static_assert(32 * kEights % kWave == 0, "a row's eights are divided evenly");
#pragma unroll
  for (uint32_t piece = 0; piece < 32 * kEights; piece += kWave) {
    const uint32_t row = (piece + lane) / kEights, eight = (piece + lane) % kEights, r = r_first + row, c = c_first + eight * 8;
    const uint32_t* from = turn + row * kPitch + eight * 8;
    typedef uint32_t four __attribute__((ext_vector_type(4)));
    const four w0 = *reinterpret_cast<const four*>(from), w1 = *reinterpret_cast<const four*>(from + 4);
    if (END == kLast) {
      float v[8];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        v[n] = __uint_as_float(w0[n]);
        v[n + 4] = __uint_as_float(w1[n]);
      }
      if (r < p.rows && c < p.cols) store_n_within<T, 8>(static_cast<T*>(p.y.p) + plane * p.y.pitch + r * p.y.ld + c, p.cols - c, v);
      continue;
    }
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
  const uint32_t r_first = w.place.r * K::kRows + wave / WC * RN * 16, c_first = w.place.c * K::kCols + wave % WC * CN * 16;
  uint32_t* turn = reinterpret_cast<uint32_t*>(lds + wave * K::kTurnBytes);
  int down_c[CN];
  constexpr bool kAhead = END != kPoly && RN * CN < 32;  // what the next rows want is on its way while these are worked on, where there are registers for it
  Found<CN> found, next;
  find_columns<CN>(p, w.plane, c_first, lane, down_c);
  if (kAhead) find_rows<END, CN>(p, w.plane, both, r_first, c_first, lane, next);
#pragma unroll
  for (int a = 0; a < RN; a += 2) {
    if (!kAhead) find_rows<END, CN>(p, w.plane, both, r_first + a * 16, c_first, lane, next);
    found = next;
    if (kAhead && a + 2 < RN) find_rows<END, CN>(p, w.plane, both, r_first + (a + 2) * 16, c_first, lane, next);
    v4f two[2][CN];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int b = 0; b < CN; ++b) two[k][b] = sum[a + k][b];
    finish_rows<T, END, CN>(p, w.plane, both, r_first + a * 16, c_first, two, found, down_c, turn, lane);
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
  const bool both = !kHalf || place.r != place.c;
  const uint32_t r_first = place.r * K::kRows + (wave / WC * RN + a) * 16, c_first = place.c * K::kCols + wave % WC * CN * 16;
  int down_c[CN];
  Found<CN> found;
  find_columns<CN>(p, plane, c_first, lane, down_c);
  find_rows<END, CN>(p, plane, both, r_first, c_first, lane, found);
  v4f sum[2][CN] = {};
  const float* from = p.part + (uint64_t)blockIdx.x * p.splits * (K::kRows * K::kCols) + wave * (RN * CN * 256) + a * CN * 256 + lane * 4;
  for (uint32_t s = 0; s < p.splits; ++s, from += K::kRows * K::kCols)
#pragma unroll
    for (int k = 0; k < 2 * CN; ++k) sum[k / CN][k % CN] += *reinterpret_cast<const v4f*>(from + k * 256);
  finish_rows<T, END, CN>(p, plane, both, r_first, c_first, sum, found, down_c, reinterpret_cast<uint32_t*>(lds + wave * K::kTurnBytes), lane);
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

// Eight numbers of binary32, as they were read into a fragment's place, as a fragment of pairs.  one: 1, which the compiler does not know: the difference and its
// rounding are one instruction then.
__device__ __forceinline__ void make_pairs(v8h (&f)[2], float one) {
  typedef float v8f __attribute__((ext_vector_type(8)));
  const v4f first = __builtin_bit_cast(v4f, f[0]), second = __builtin_bit_cast(v4f, f[1]);
  const v8f x = __builtin_shufflevector(first, second, 0, 1, 2, 3, 4, 5, 6, 7);
  f[0] = __builtin_convertvector(x, v8h);
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    const v2h low = rounded(rest_of(x[k], one, f[0][k]), rest_of(x[k + 1], one, f[0][k + 1]));
    f[1][k] = low[0];
    f[1][k + 1] = low[1];
  }
}

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
  // Where a lane reads its rows' pieces; the low parts (of binary32 the other four of eight) are four pieces on.
  constexpr bool kFloats = END == kApply || END == kLast;
  float one = 1.f;
  if (kFloats) asm("" : "+v"(one));
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
  for (int k = 0; k < CN; ++k) {
    read_b(even, k, 0);
    if (kFloats) make_pairs(even.b[k], one);
  }
  uint32_t slot = 0;
  auto stage = [&](Fragments& now, Fragments& then) {
    const uint32_t next = slot + K::kStageBytes == K::kRing ? 0u : slot + K::kStageBytes;
    wait_and_meet<(SLOTS - 2) * K::kLoads>();  // this stage is in registers everywhere, and the next one in LDS
    __builtin_amdgcn_sched_barrier(0);
    // (what is to become pairs is read with the first group)
    constexpr int kReads = kFloats ? CN : (CN + RN - 1) / RN, kAsks = (K::kLoads + RN - 1) / RN, kMakes = (CN + RN - 2) / (RN - 1);
#pragma unroll
    for (int g = 0; g < RN; ++g) {
      read_a(then, g, next);
#pragma unroll
      for (int k = g * kReads; k < (g + 1) * kReads && k < CN; ++k) read_b(then, k, next);
#pragma unroll
      for (int j = g * kAsks; j < (g + 1) * kAsks && j < K::kLoads; ++j) of.load(j, slot);
      if (kFloats && g > 0) {
#pragma unroll
        for (int k = (g - 1) * kMakes; k < g * kMakes && k < CN; ++k) make_pairs(then.b[k], one);
      }
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
// of the last two groups; the others follow the first groups of the next stage.  (256 x 256 with one, two and four, of pairs on both sides: 306, 288, 291 us for a product of 4096 x 4096.)
// E X of 4096 x 4096 takes 323 us, 1.28 PFLOP/s of products of 16 bits, 63 % of the matrix units' time at 1.89 GHz (the library's product of binary16 makes 1.26);
// with X as pairs in memory it would be 294, but then binary32 has to be read and written beside them, which makes 341.  Half of X X^T, by tiles of 192, 183.
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
  constexpr bool kFloats = END == kApply || END == kLast;
  float one = 1.f;
  if (kFloats) asm("" : "+v"(one));
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
  for (int k = 0; k < CN; ++k) {
    read_b(0, k, 0);
    if (kFloats && k < CN / kAhead) make_pairs(b[0][k], one);
  }
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
      if (kFloats && g == 0) {
#pragma unroll
        for (int k = CN / kAhead; k < CN; ++k) make_pairs(b[set][k], one);
      }
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
      if (kFloats && g == kMeet + 1) {
#pragma unroll
        for (int k = 0; k < CN / kAhead; ++k) make_pairs(b[1 - set][k], one);
      }
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

// How a product is made: whatever tiles, and pieces of the tiles that would have the chip to themselves at the end, an estimate of the time says.  (Five
// steps with one kind of tile, us: 4096 x 4096 with 256, 192, 128 and 64: 4070, 3690, 4490, 5290, and 3470 by the estimate; 256 x 4096: 1490, 920, 510, 270,
// the last in pieces 175.)
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
// A wavefront holds CT tiles of 16 columns of X in binary32, all NT of their tiles of rows, as its matrix instructions leave them: four consecutive rows of a
// column a lane.  E X takes them from there, as pairs: which of E's columns meets which of X's rows in a lane's eight is free as long as both sides agree, so a
// lane's two fours of rows are its eight, and E's are read from LDS in that order.  Only X X^T wants rows of X, through LDS, where a word is a pair.
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

// What both kernels do; all of a workgroup come to each of these as often as the others.
template <int NT, int CT>
struct Small {
  static_assert(NT % 2 == 0, "a lane's eight are two tiles' fours");
  static constexpr int kRows = NT * 16, kCols = CT * 16 * kSmallWaves, kPitch = kCols + 4, kSquare = kRows + 4, kTiles = NT * (NT + 1) / 2;
  static constexpr int kMine = (kTiles + kSmallWaves - 1) / kSmallWaves;
  typedef uint32_t four __attribute__((ext_vector_type(4)));
  typedef v4f Strip[NT][CT];
  typedef v8h Fragments[NT / 2][CT];
  uint32_t *of_x, *of_p;  // LDS: [kRows][kPitch]; [kRows][kSquare], G, then E
  uint32_t lane, wave, i, g, r_in;

  __device__ __forceinline__ Small(uint32_t* x, uint32_t* p) : of_x(x), of_p(p) {
    lane = threadIdx.x % kWave;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    i = lane % 16;
    g = lane / 16;
    r_in = g * 4;
  }
  // Addresses that a loop's body would keep in registers from turn to turn are made again instead.
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(lane), "+v"(i), "+v"(g), "+v"(r_in)); }
  // What rows are held times, of a step (LDS: [kRows]), for a lane's four of a tile.
  __device__ __forceinline__ v4f rows_up(const float* up, uint32_t tile) const { return *reinterpret_cast<const v4f*>(up + tile * 16 + r_in); }
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

  // p of a lane's columns.
  __device__ __forceinline__ void columns_down(const Strip& x, int (&down)[CT]) const {
#pragma unroll
    for (int b = 0; b < CT; ++b) {
      float sum = 0.f;
#pragma unroll
      for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += x[a][b][k] * x[a][b][k];
      sum += __shfl_xor(sum, 16, kWave);
      sum += __shfl_xor(sum, 32, kWave);
      down[b] = down_of(sqrtf(sum));
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // X as pairs in LDS, and as fragments.
  __device__ __forceinline__ void to_lds(const Strip& x, const float* up) const {
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      const v4f rows = rows_up(up, a);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int b = 0; b < CT; ++b) of_x[(a * 16 + r_in + k) * kPitch + column(b)] = pair_of(x[a][b][k], rows[k]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // Both at once, where rows and columns are held alike.
  __device__ __forceinline__ void to_both(const Strip& x, float up, Fragments& high, Fragments& low) const {
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
      for (int b = 0; b < CT; ++b) {
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          v2h h, l;
          split(x[a][b][k], x[a][b][k + 1], up, up, h, l);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            high[a / 2][b][a % 2 * 4 + k + n] = h[n];
            low[a / 2][b][a % 2 * 4 + k + n] = l[n];
            of_x[(a * 16 + r_in + k + n) * kPitch + column(b)] = __builtin_bit_cast(uint32_t, (v2h{h[n], l[n]}));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  __device__ __forceinline__ void divide(const Strip& x, const int (&down)[CT], int c, Fragments& high, Fragments& low) const {
#pragma unroll
    for (int b = 0; b < CT; ++b) {
      const float up = two_to(held(down[b], c));
#pragma unroll
      for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          v2h h, l;
          split(x[a][b][k], x[a][b][k + 1], up, up, h, l);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            high[a / 2][b][a % 2 * 4 + k + n] = h[n];
            low[a / 2][b][a % 2 * 4 + k + n] = l[n];
          }
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The tile of a number: rows first, c <= r.
  static __device__ __forceinline__ Place place(uint32_t number) {
    uint32_t row = 0;
    while (number > row) number -= ++row;
    return Place{row, number};
  }
  // A tile as rows of r and as rows of c hold it, each times its powers.
  __device__ __forceinline__ void put(const Place& at, const v4f& by_r, const v4f& by_c, const v4f& up_r, const v4f& up_c) const {
    four pair;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      of_p[(at.r * 16 + r_in + k) * kSquare + at.c * 16 + i] = pair_of(by_r[k], up_r[k]);
      pair[k] = pair_of(by_c[k], up_c[k]);
    }
    if (at.r != at.c) *reinterpret_cast<four*>(of_p + (at.c * 16 + i) * kSquare + at.r * 16 + r_in) = pair;
  }
  // One of sums, which are times both rows' powers, of rows and of column.
  __device__ __forceinline__ void put_sums(const Place& at, const v4f& sum, const v4f& rows, float column) const {
    const float less = inverse_two(column);
    v4f less_r;
#pragma unroll
    for (int k = 0; k < 4; ++k) less_r[k] = inverse_two(rows[k]);
    put(at, sum, sum, v4f{less, less, less, less}, less_r);
  }
  // A tile of X X^T, of what is in LDS.
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
  // E, in the place of G.
  __device__ __forceinline__ void polynomial(float times, float square, const float* up, int u) const {
    const float unit = two_to(-u);
    v4f by_r[kMine], by_c[kMine];
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const uint32_t t = wave + n * kSmallWaves;
      if (t >= kTiles) continue;
      const Place at = place(t);
      const v4f rows = rows_up(up, at.r);
      const float column = up[at.c * 16 + i];
      const four turned = *reinterpret_cast<const four*>(of_p + (at.c * 16 + i) * kSquare + at.r * 16 + r_in);
      four straight;
#pragma unroll
      for (int k = 0; k < 4; ++k) straight[k] = of_p[(at.r * 16 + r_in + k) * kSquare + at.c * 16 + i];
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
      const float less = square * inverse_two(column);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        by_r[n][k] = __builtin_fmaf(all[k], less, times * value_of(straight[k]));
        by_c[n][k] = __builtin_fmaf(all[k], square * inverse_two(rows[k]), times * value_of(turned[k]));
      }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const uint32_t t = wave + n * kSmallWaves;
      if (t < kTiles) put(place(t), by_r[n], by_c[n], v4f{unit, unit, unit, unit}, v4f{unit, unit, unit, unit});
    }
    __syncthreads();
  }

  // a X + E X, in the place of X.
  __device__ __forceinline__ void apply(const Fragments& high, const Fragments& low, const int (&down)[CT], float plus, const float* up, int c, int u, Strip& x) const {
    float less[CT];
#pragma unroll
    for (int b = 0; b < CT; ++b) less[b] = two_to(u - held(down[b], c));
#pragma unroll
    for (int a = 0; a < NT; ++a) {
      v4f all[CT] = {};
      const v4f rows = rows_up(up, a);
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
      for (int k = 0; k < 4; ++k) {
        const float unit = inverse_two(rows[k]);
#pragma unroll
        for (int b = 0; b < CT; ++b) x[a][b][k] = __builtin_fmaf(all[b][k], unit * less[b], plus * x[a][b][k]);
      }
    }
  }
  __device__ __forceinline__ void times(float scale, Strip& x) const {
#pragma unroll
    for (int k = 0; k < NT * CT; ++k)
#pragma unroll
      for (int n = 0; n < 4; ++n) x[k / CT][k % CT][n] *= scale;
  }
};

// The sum over the 16 lanes of a row, in each of them.
__device__ __forceinline__ float row_of_16_sum(float x) {
  x = plus_other<0xB1, 0xF>(x);
  x = plus_other<0x4E, 0xF>(x);
  x = plus_other<0x141, 0xF>(x);
  return plus_other<0x140, 0xF>(x);
}

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
  Step step[kSmallSteps];
};

// 16 x 64 x 256 in five steps: 32 us: a step is four meetings, and in between ten tiles of G and of E for eight wavefronts, one chain of instructions each.  (Three
// launches a step took 80.)
template <int NT, int CT>
__global__ void __launch_bounds__(kSmallWaves* kWave) small_kernel(SmallTask p) {
  using K = Small<NT, CT>;
  __shared__ __align__(16) uint32_t of_x[K::kRows * K::kPitch];
  __shared__ __align__(16) uint32_t of_p[K::kRows * K::kSquare];
  __shared__ __align__(16) float ups[2][K::kRows];  // what rows are held times, of this step and the next one
  __shared__ double of_wave[kSmallWaves];
  K all(of_x, of_p);
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
  // p of the columns, which a wavefront has whole, and of the rows, joined in X's place
  int down[CT];
  all.columns_down(x, down);
  float(*of_rows)[K::kRows] = reinterpret_cast<float(*)[K::kRows]>(of_x);
#pragma unroll
  for (int a = 0; a < NT; ++a)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float squares = 0.f;
#pragma unroll
      for (int b = 0; b < CT; ++b) squares += x[a][b][k] * x[a][b][k];
      squares = row_of_16_sum(squares);
      if (all.i == 0) of_rows[all.wave][a * 16 + all.r_in + k] = squares;
      __builtin_amdgcn_sched_barrier(0);
    }
  __syncthreads();
  // Rows whose norms are within 2^kEven are all held as the longest one is (what that takes from the others' ends, ten bits of 39, no sum shows), and so are a
  // wavefront's columns, none of which has an element above that: one division of X makes rows and fragments then.  Each wavefront looks at all rows for itself.
  // (16 x 64 x 256 32 us, and with two divisions 34.)
  constexpr int kEven = 10, kTop = 127;
  int down_row[2], longest = 0, shortest = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t r = all.lane + h * kWave;
    down_row[h] = 0;
    if (h * kWave >= K::kRows || r >= K::kRows) continue;
    float squares = 0.f;
    for (int k = 0; k < kSmallWaves; ++k) squares += of_rows[k][r];
    down_row[h] = down_of(sqrtf(squares));
    if (r < p.n) {
      longest = max(longest, kTop - down_row[h]);
      shortest = max(shortest, down_row[h]);
    }
  }
  longest = kTop - (int)wave_max_bits((uint32_t)longest);
  shortest = (int)wave_max_bits((uint32_t)shortest);
  const bool even = shortest - longest <= kEven;
  int of_columns = 0;
#pragma unroll
  for (int b = 0; b < CT; ++b) of_columns = max(of_columns, down[b]);
  const bool alike = even && (int)wave_max_bits((uint32_t)of_columns) - longest <= kEven;
#pragma unroll
  for (int b = 0; b < CT; ++b) down[b] = alike ? longest : down[b];
  const int row = even ? longest : down_row[all.wave % 2];
  if (threadIdx.x < K::kRows) ups[0][threadIdx.x] = two_to(held(row, p.step[0].before));
  __syncthreads();
  for (uint32_t k = 0; k < p.steps; ++k) {
    const Step step = p.step[k];
    const float* up = ups[k % 2];
    all.again();
    typename K::Fragments high, low;
    if (alike)
      all.to_both(x, two_to(held(longest, step.before)), high, low);
    else
      all.to_lds(x, up);
    __syncthreads();
    if (threadIdx.x < K::kRows) ups[1 - k % 2][threadIdx.x] = two_to(held(row, step.after));
#pragma unroll 1
    for (uint32_t t = all.wave; t < K::kTiles; t += kSmallWaves) {
      const Place at = K::place(t);
      const v4f rows = all.rows_up(up, at.r);
      const float column = up[at.c * 16 + all.i];
      all.put_sums(at, all.gram(at), rows, column);
    }
    __syncthreads();
    all.polynomial(step.b, step.c, up, step.poly);
    if (!alike) all.divide(x, down, step.before, high, low);
    all.apply(high, low, down, step.a, up, step.before, step.poly, x);
  }
  all.times(p.scale, x);
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
  Step done;           // of step - 1
  int after;           // c of this step
  const double *part, *by_n;  // squares: [matrix][parts], and of X's rows, [matrix][counts][n]
  uint32_t parts, counts;
  int32_t *of_row, *of_col;  // p: [matrix][96 at most], [matrix][strip][columns]
  float* state;               // [matrix][strip][tile of rows][tile of columns][thread][4]: X, from step 1 on
  const float* sums;          // [matrix][strip][tile of X X^T][lane][4], from the launch before
  float* next;                // the same for the next one
};

// A strip of columns in one step: X X^T from what all strips found of it, E, by every workgroup for itself, a X + E X, and this strip's part of the next X X^T.
// Latencies bound it: 64 x 1024 in five steps is seven launches of 5 to 8 us, where tiles take three a step and more.
template <int NT, int CT>
__global__ void __launch_bounds__(kSmallWaves* kWave) strip_kernel(StripTask p) {
  using K = Small<NT, CT>;
  __shared__ __align__(16) uint32_t of_x[K::kRows * K::kPitch];
  __shared__ __align__(16) uint32_t of_p[K::kRows * K::kSquare];
  __shared__ __align__(16) float ups[2][K::kRows];  // what rows are held times, of the step that is done and of the next one
  const K all(of_x, of_p);
  const uint32_t m = blockIdx.y, strip = blockIdx.x, strips = gridDim.x;
  const uint32_t c0 = strip * K::kCols, left = p.m - c0;
  typename K::Strip x;
  int down[CT];
  float* state = p.state + ((uint64_t)m * strips + strip) * (K::kRows * K::kCols) + threadIdx.x * 4;
  int32_t *rows = p.of_row + (uint64_t)m * K::kRows, *columns = p.of_col + ((uint64_t)m * strips + strip) * K::kCols;
  if (p.step <= 1) {
    with_type(p.of_x, [&](auto of) {
      using T = decltype(of);
      all.load(static_cast<const T*>(p.x.p) + m * p.x.pitch + c0 * (p.tall ? p.x.ld : 1), p.tall, p.x.ld, p.n, left, x);
    });
    const double inverse = inverse_of(sum_of_parts(p.part + (uint64_t)m * p.parts, p.parts, all.lane), p.eps);
    all.scale(inverse, p.n, left, x);
    if (p.step == 0) {
      // p of the rows by every strip for itself, 64 at a time by 256 lanes; the first strip leaves them for the launches that follow
      auto joined = reinterpret_cast<double(*)[4][kWave]>(of_x);
      const uint32_t half = threadIdx.x / kBlock, t = threadIdx.x % kBlock, at = half * kWave + t % kWave;
      const int row = down_of_sums(p.by_n + (uint64_t)m * p.counts * p.n, p.counts, p.n, half * kWave, inverse, joined[half], t);
      if (t < kWave && at < K::kRows) {
        ups[1][at] = two_to(held(row, p.after));
        if (strip == 0) rows[at] = row;
      }
      all.columns_down(x, down);
#pragma unroll
      for (int b = 0; b < CT; ++b)
        if (all.g == 0) columns[all.column(b)] = down[b];
      __syncthreads();
    }
  } else {
#pragma unroll
    for (int k = 0; k < NT * CT; ++k) x[k / CT][k % CT] = *reinterpret_cast<const v4f*>(state + k * (kSmallWaves * kWave * 4));
  }
  if (p.step > 0) {
    if (threadIdx.x < K::kRows) {
      ups[0][threadIdx.x] = two_to(held(rows[threadIdx.x], p.done.before));
      ups[1][threadIdx.x] = two_to(held(rows[threadIdx.x], p.after));
    }
#pragma unroll
    for (int b = 0; b < CT; ++b) down[b] = columns[all.column(b)];
    __syncthreads();
    const float* sums = p.sums + (uint64_t)m * strips * (K::kTiles * 256) + all.lane * 4;
#pragma unroll 1
    for (uint32_t t = all.wave; t < K::kTiles; t += kSmallWaves) {
      const Place at = K::place(t);
      const v4f rows = all.rows_up(ups[0], at.r);
      const float column = ups[0][at.c * 16 + all.i];
      v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (uint32_t k = 0; k < strips; ++k) sum += *reinterpret_cast<const v4f*>(sums + ((uint64_t)k * K::kTiles + t) * 256);
      all.put_sums(at, sum, rows, column);
    }
    __syncthreads();
    all.polynomial(p.done.b, p.done.c, ups[0], p.done.poly);
    typename K::Fragments high, low;
    all.divide(x, down, p.done.before, high, low);
    all.apply(high, low, down, p.done.a, ups[0], p.done.before, p.done.poly, x);
    if (p.step == p.steps) {
      all.times(p.scale, x);
      with_type(p.of_y, [&](auto of) {
        using T = decltype(of);
        all.store(static_cast<T*>(p.y.p) + m * p.y.pitch + c0 * (p.tall ? p.y.ld : 1), p.tall, p.y.ld, p.n, left, x);
      });
      return;
    }
#pragma unroll
    for (int k = 0; k < NT * CT; ++k) *reinterpret_cast<v4f*>(state + k * (kSmallWaves * kWave * 4)) = x[k / CT][k % CT];
  }
  all.to_lds(x, ups[1]);
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
// steps, us, and by tiles: 64 x 1024 49 and 112, 32 x 4096 38 and 120, 64 x 8192 91 and 146, 100 x 64 x 1024 168 and 232, 100 x 64 x 8000 840 and 1360, with up to
// 32 strips 82 of 64 x 8192 and 1310 of the last; 96 x 1000 73 and 114, 64 x 96 x 1000 212 and 222, 300 x 70 x 300 305 and 331, but 100 x 96 x 2000 645 and 514, so
// of more than 64 rows not where the chip is full several times anyway.)
constexpr uint32_t kMostStrips = 16;
uint32_t strip_of(const Extent& e) {
  const uint64_t n = std::min(e.rows, e.cols), m = std::max(e.rows, e.cols);
  const uint32_t most = n <= 64 ? 512 : n <= 96 ? 256 : 0;  // (LDS has room for no more)
  for (uint32_t cols = 128; cols <= most; cols *= 2) {
    const uint64_t strips = (m + cols - 1) / cols;
    if (strips <= kMostStrips) return n <= 64 || e.workers * strips <= 4 * kCus ? cols : 0;
  }
  return 0;
}

// How a matrix is taken for its norms.
struct Norms {
  uint32_t lanes, chunks, strips;
  double *part, *by_row, *by_col;
};
template <typename F>
Norms norms_of(const Extent& e, F take) {
  Norms l{};
  l.lanes = 1;
  while (l.lanes < kWave && l.lanes * 8 < e.cols) l.lanes *= 2;
  l.chunks = (uint32_t)((e.cols + kChunk - 1) / kChunk);
  // (four turns of a workgroup at least.  What strips have of a column is joined: of twice as many 4 x 2053 x 1003 bfloat16 takes 12 us instead of 15 here, and 7.5
  // instead of 5 there; 4096 x 4096 20 and 21, 10.4 and 6.8.)
  const uint64_t turns = (e.rows + 16 * (kWave / l.lanes) - 1) / (16 * (kWave / l.lanes));
  l.strips = (uint32_t)std::min<uint64_t>({std::max<uint64_t>(1, 1024 / (e.workers * (uint64_t)l.chunks)), turns, 64});
  l.part = static_cast<double*>(take(e.workers * (uint64_t)l.chunks * l.strips * sizeof(double)));
  l.by_row = static_cast<double*>(take(e.workers * (uint64_t)l.chunks * e.rows * sizeof(double)));
  l.by_col = static_cast<double*>(take(e.workers * (uint64_t)l.strips * e.cols * sizeof(double)));
  return l;
}

struct Strips {
  uint64_t n, m;
  uint32_t cols, count;
  Norms norms;
  int32_t *of_row, *of_col;
  float *state, *sums[2];
  uint64_t bytes;
};
Strips strips_of(const Extent& e, char* scratch) {
  Strips l{};
  l.n = std::min(e.rows, e.cols);
  l.m = std::max(e.rows, e.cols);
  l.cols = strip_of(e);
  l.count = (uint32_t)((l.m + l.cols - 1) / l.cols);
  auto take = [&](uint64_t bytes) -> void* {
    char* here = scratch + l.bytes;
    l.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  const uint64_t tiles = (l.n + 31) / 32 * 2, all = e.workers * (uint64_t)l.count;
  l.norms = norms_of(e, take);
  l.of_row = static_cast<int32_t*>(take(e.workers * tiles * 16 * sizeof(int32_t)));
  l.of_col = static_cast<int32_t*>(take(all * l.cols * sizeof(int32_t)));
  l.state = static_cast<float*>(take(all * tiles * 16 * l.cols * sizeof(float)));
  for (float*& sums : l.sums) sums = static_cast<float*>(take(all * (tiles * (tiles + 1) / 2 * 256) * sizeof(float)));
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
  Norms norms;
  int32_t *of_n, *of_m;  // p of X's rows and columns
  Pairs x_by_n, gram, poly;
  Rows x_turned[2], gram_floats;
  float* sums;  // of tiles that are made in pieces
  uint64_t bytes;
};

Layout layout_of(const Extent& e, char* scratch) {
  Layout l{};
  l.tall = e.rows > e.cols;
  l.n = std::min(e.rows, e.cols);
  l.m = std::max(e.rows, e.cols);
  auto take = [&](uint64_t bytes) -> void* {
    char* here = scratch + l.bytes;
    l.bytes += (bytes + 255) / 256 * 256;
    return here;
  };
  auto pairs = [&](uint64_t rows, uint64_t cols) {
    const uint64_t ld = pair_row(cols);
    return Pairs{static_cast<char*>(take(e.workers * rows * ld)), ld, rows * ld};
  };
  l.norms = norms_of(e, take);
  l.of_n = static_cast<int32_t*>(take(e.workers * downs(l.n) * sizeof(int32_t)));
  l.of_m = static_cast<int32_t*>(take(e.workers * downs(l.m) * sizeof(int32_t)));
  l.x_by_n = pairs(l.n, l.m);
  for (Rows& x : l.x_turned) x = pairs(l.m, l.n);
  l.gram = pairs(l.n, l.n);
  l.gram_floats = pairs(l.n, l.n);
  l.poly = pairs(l.n, l.n);
  const uint32_t n = (uint32_t)l.n, m = (uint32_t)l.m, n_stages = (n + kBlockCols - 1) / kBlockCols, m_stages = (m + kBlockCols - 1) / kBlockCols;
  l.sums = static_cast<float*>(take(std::max({part_bytes(plan_of(true, n, n, e.workers, m_stages)), part_bytes(plan_of(true, n, n, e.workers, n_stages)),
                                              part_bytes(plan_of(false, n, m, e.workers, n_stages))})));
  return l;
}

void launch_norms(tng_type type, const Extent& e, const View& x, const Norms& l, hipStream_t s) {
  const NormsTask p{e.rows, e.cols, x, l.lanes, l.chunks, l.strips, l.part, l.by_row, l.by_col};
  const dim3 grid(l.chunks * l.strips, e.workers);
  switch (type) {
    case TNG_TYPE_F32: norms_kernel<float><<<grid, kBlock, 0, s>>>(p); break;
    case TNG_TYPE_BF16: norms_kernel<bf16_t><<<grid, kBlock, 0, s>>>(p); break;
    default: norms_kernel<f16_t><<<grid, kBlock, 0, s>>>(p); break;
  }
}
void launch_start(tng_type type, uint32_t workers, const StartTask& p, hipStream_t s) {
  const dim3 grid((uint32_t)((p.cols + kTurn - 1) / kTurn), (uint32_t)((p.rows + kTurn - 1) / kTurn), workers);
  switch (type) {
    case TNG_TYPE_F32: start_kernel<float><<<grid, kBlock, 0, s>>>(p); break;
    case TNG_TYPE_BF16: start_kernel<bf16_t><<<grid, kBlock, 0, s>>>(p); break;
    default: start_kernel<f16_t><<<grid, kBlock, 0, s>>>(p); break;
  }
}

}  // namespace

// The largest |s p(s^2)|, |p(s^2)| and |s (b + c s^2)| s of s in 0 .. top, p(t) = a + b t + c t^2: at the ends, or where a derivative is 0.
static void reach(const float* abc, double top, double* of_x, double* of_p, double* of_e) {
  const double a = abc[0], b = abc[1], c = abc[2], end = top * top;
  auto p = [&](double t) { return std::fabs(a + t * (b + t * c)); };
  auto e = [&](double t) { return std::sqrt(t) * std::fabs(b + t * c); };
  *of_p = std::max(p(0.), p(end));
  *of_x = std::sqrt(end) * p(end);
  *of_e = e(end);
  auto at = [&](double t) {
    if (!(t > 0. && t < end)) return;
    *of_p = std::max(*of_p, p(t));
    *of_x = std::max(*of_x, std::sqrt(t) * p(t));
    *of_e = std::max(*of_e, e(t));
  };
  at(-b / (2. * c));
  const double root = 9. * b * b - 20. * a * c;  // of a + 3 b t + 5 c t^2
  if (root >= 0.) {
    at((-3. * b + std::sqrt(root)) / (10. * c));
    at((-3. * b - std::sqrt(root)) / (10. * c));
  }
  at(-a / (3. * b));  // (c = 0)
  at(-b / (3. * c));  // of b + 3 c t
}

// The steps with their powers of two: norms of X's rows grow by the largest |p|, those of E's are those of X's times the largest |s (b + c s^2)|, which held at
// 2^(15 - u) stay below binary16's end.  False where singular values reach 2, or |p| 8.  (Rounding may add to both: 0.1 %.)
static bool steps_of(const float* coefficients, uint32_t steps, Step* out) {
  double top = 1., grown = 0.;
  auto whole = [](double v, double low, double high) { return (int)std::ceil(std::min(std::max(v, low), high)); };
  for (uint32_t k = 0; k < steps; ++k) {
    const float* abc = coefficients + 3 * k;
    double of_x, of_p, of_e;
    reach(abc, top, &of_x, &of_p, &of_e);
    if (!(of_p < 7.9)) return false;
    top = of_x * 1.001;
    if (!(top < 1.98)) return false;
    if (out == nullptr) continue;
    const int before = whole(grown, 0., 127.);
    grown += std::log2(std::max(of_p, 1e-30) * 1.001);
    out[k] = Step{abc[0], abc[1], abc[2], before, whole(grown, 0., 127.), whole(std::log2(std::max(of_e, 1e-30) * 1.001 / 1.99), -40., 40.)};
  }
  return true;
}

bool orthogonal_in_range(const float* coefficients, uint32_t steps) { return steps_of(coefficients, steps, nullptr); }

size_t orthogonal_bytes(const Extent& e) {
  const uint64_t n = std::min(e.rows, e.cols), m = std::max(e.rows, e.cols);
  return is_small(n, m) ? 0 : strip_of(e) != 0 ? strips_of(e, nullptr).bytes : layout_of(e, nullptr).bytes;
}

hipError_t launch_orthogonalize(tng_type of_x, tng_type of_y, const Extent& e, const View& x, const float* coefficients, uint32_t steps, float eps, float scale,
                                const View& y, char* scratch, hipStream_t s) {
  const uint64_t short_side = std::min(e.rows, e.cols), long_side = std::max(e.rows, e.cols);
  SmallTask small{(uint32_t)short_side, (uint32_t)long_side, steps, e.rows > e.cols, x, y, of_x, of_y, eps, scale, {}};
  const Step* const step = small.step;
  steps_of(coefficients, steps, small.step);
  if (is_small(short_side, long_side)) return launch_small(small, e.workers, s);
  if (strip_of(e) != 0) {
    const Strips l = strips_of(e, scratch);
    launch_norms(of_x, e, x, l.norms, s);
    const bool tall = e.rows > e.cols;
    StripTask p{(uint32_t)l.n, (uint32_t)l.m, 0, steps, tall, x, y, of_x, of_y, eps, scale, {}, 0, l.norms.part, tall ? l.norms.by_col : l.norms.by_row,
                l.norms.chunks * l.norms.strips, tall ? l.norms.strips : l.norms.chunks, l.of_row, l.of_col, l.state, nullptr, nullptr};
    for (; p.step <= steps; ++p.step) {
      if (p.step > 0) p.done = step[p.step - 1];
      p.after = p.done.after;
      p.sums = l.sums[(p.step + 1) % 2];
      p.next = l.sums[p.step % 2];
      launch_strip(p, l, e.workers, s);
    }
    return hipGetLastError();
  }
  const Layout l = layout_of(e, scratch);
  launch_norms(of_x, e, x, l.norms, s);
  int32_t *const of_row = l.tall ? l.of_m : l.of_n, *const of_col = l.tall ? l.of_n : l.of_m;
  const DownTask down{e.rows, e.cols, l.norms.chunks, l.norms.strips, l.norms.part, l.norms.by_row, l.norms.by_col, eps, of_row, of_col};
  downs_kernel<<<dim3((uint32_t)((downs(e.rows) + downs(e.cols)) / kWave), e.workers), kBlock, 0, s>>>(down);
  launch_start(of_x, e.workers,
               StartTask{e.rows, e.cols, x, l.norms.part, l.norms.chunks * l.norms.strips, eps, l.tall, of_row, of_col, l.x_by_n, l.x_turned[0]}, s);
  const uint32_t n = (uint32_t)l.n, m = (uint32_t)l.m, n_stages = (n + kBlockCols - 1) / kBlockCols, m_stages = (m + kBlockCols - 1) / kBlockCols;
  for (uint32_t k = 0; k < steps; ++k) {
    PairTask gram{};
    gram.rows = gram.cols = n;
    gram.stages = m_stages;
    gram.planes = e.workers;
    gram.a = gram.b = l.x_by_n;
    gram.of_r = gram.of_c = l.of_n;
    gram.pitch_r = gram.pitch_c = downs(l.n);
    gram.before = step[k].before;
    gram.after = step[k].after;
    gram.poly = step[k].poly;
    gram.gram = l.gram_floats;
    gram.plus = step[k].a;
    gram.times = step[k].b;
    gram.square = step[k].c;
    gram.by_r = gram.by_c = l.gram;
    gram.part = l.sums;
    product<float, kGram>(gram, s);
    PairTask poly = gram;
    poly.stages = n_stages;
    poly.a = poly.b = l.gram;
    poly.by_r = poly.by_c = l.poly;
    product<float, kPoly>(poly, s);
    PairTask apply = poly;
    apply.cols = m;
    apply.a = l.poly;
    apply.b = l.x_turned[k % 2];
    apply.of_c = l.of_m;
    apply.pitch_c = downs(l.m);
    apply.by_r = l.x_by_n;
    apply.x_then = l.x_turned[1 - k % 2];
    apply.tall = l.tall;
    apply.y = y;
    apply.scale = scale;
    if (k + 1 < steps) {
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
