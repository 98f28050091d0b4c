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

// 64 x 64 elements of x for a workgroup: as pairs along the columns, and turned, along the rows.
constexpr uint32_t kTurn = 64;

template <typename T>
__global__ void __launch_bounds__(kBlock) start_kernel(StartTask p) {
  __shared__ uint32_t tile[kTurn][kTurn + 1];  // [row][column]: a pair
  __shared__ double inverse;
  const uint32_t m = blockIdx.z;
  if (threadIdx.x < kWave) {
    double sum = 0.;
    for (uint32_t k = threadIdx.x; k < p.parts; k += kWave) sum += p.part[(uint64_t)m * p.parts + k];
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
    // (a matrix that holds what is not finite is NaN as a whole)
    if (threadIdx.x == 0) inverse = sum < __builtin_inf() ? 1. / (sqrt(sum) + (double)p.eps) : __builtin_nan("");
  }
  __syncthreads();
  const double inv = inverse * (double)kOfX;
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

// A wavefront makes RN x CN tiles of 16 x 16 results, WR x WC of them a workgroup's tile.  A stage is 32 columns of the operands' rows, 128 bytes each; SLOTS of them lie
// in LDS.  While the products of a stage run, the next one's fragments are read into registers, and the loads of the stage that follows the last one in LDS
// are asked for, in the place of the one that has been read: one wait and one barrier a stage.
template <int RN, int CN, int WR, int WC, int SLOTS>
struct PairKernel {
  static constexpr int kRows = RN * WR * 16, kCols = CN * WC * 16, kWaves = WR * WC, kThreads = kWaves * kWave;
  static constexpr int kStageBytes = (kRows + kCols) * 128, kRing = SLOTS * kStageBytes;
  static constexpr int kLoads = (kRows + kCols) / 8 / kWaves, kLoadsOfA = kRows / 8 / kWaves;
  static_assert(kRows % (8 * kWaves) == 0 && kCols % (8 * kWaves) == 0, "loads divide evenly");
  // Behind the stages: the results of 32 rows of each wavefront at a time, turned.  (Four words more a row: a wavefront's four groups of rows meet in no bank.)
  static constexpr int kTurnPitch = CN * 16 + 4, kTurnBytes = 32 * kTurnPitch * 4;
  static_assert(RN % 2 == 0 && kTurnBytes * kWaves <= kRing, "results are turned in the stages' place");
};

template <typename T, int END, int RN, int CN, int WR, int WC, int SLOTS>
__global__ void __launch_bounds__(WR* WC* kWave) pair_kernel(PairTask p) {
  using K = PairKernel<RN, CN, WR, WC, SLOTS>;
  constexpr bool kHalf = END == kGram || END == kPoly;
  __shared__ __align__(1024) char lds[K::kRing];
  const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wr = wave / WC, wc = wave % WC;
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
  const uint32_t down = (p.rows + K::kRows - 1) / K::kRows, across = (p.cols + K::kCols - 1) / K::kCols;
  const uint32_t each = kHalf ? down * (down + 1) / 2 : down * across, number = number_of(blockIdx.x, each * p.planes), plane = number / each;
  const Place place = place_of<kHalf>(number - plane * each, down, across);
  const uint32_t r0 = place.r * K::kRows, c0 = place.c * K::kCols;

  // number j of a wavefront's loads takes 8 rows, a row eight lanes; past the last stage nothing is read, and what the loads clear is not looked at
  uint64_t base_a = reinterpret_cast<uint64_t>(p.a.p) + plane * p.a.pitch + r0 * p.a.ld, base_b = reinterpret_cast<uint64_t>(p.b.p) + plane * p.b.pitch + c0 * p.b.ld;
  const uint32_t rows = min(p.rows - r0, (uint32_t)K::kRows), cols = min(p.cols - c0, (uint32_t)K::kCols);
  uint32_t bytes_a = (rows - 1) * (uint32_t)p.a.ld + p.stages * 128u, bytes_b = (cols - 1) * (uint32_t)p.b.ld + p.stages * 128u;
  uint32_t offset[K::kLoads];
#pragma unroll
  for (int j = 0; j < K::kLoads; ++j) {
    const bool of_a = j < K::kLoadsOfA;
    const uint32_t r = ((of_a ? j : j - K::kLoadsOfA) * K::kWaves + wave) * 8 + lane / 8;
    offset[j] = min(r, (of_a ? rows : cols) - 1) * (uint32_t)(of_a ? p.a.ld : p.b.ld) + (lane % 8 ^ (r >> 1 & 7u)) * 16;
  }
  int ahead = (int)p.stages;  // stages not asked for
  auto load_one = [&](int j, uint32_t slot) {
    const bool of_a = j < K::kLoadsOfA;
    load_to_lds(of_a ? base_a : base_b, ahead > 0 ? (of_a ? bytes_a : bytes_b) : 0u, offset[j], lds0 + slot + (j * K::kWaves + wave) * 1024);
  };
  auto asked_one = [&]() {
    --ahead;
    base_a += 128;
    base_b += 128;
    bytes_a -= 128;
    bytes_b -= 128;
  };

  // Where a lane reads its rows' pieces; the low parts are four pieces on.
  const uint32_t i = lane % 16;
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
    for (int j = 0; j < K::kLoads; ++j) load_one(j, k * K::kStageBytes);
    asked_one();
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
      for (int j = g * kAsks; j < (g + 1) * kAsks && j < K::kLoads; ++j) load_one(j, slot);
#pragma unroll
      for (int b = 0; b < CN; ++b) sum[g][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.a[g][0], now.b[b][1], sum[g][b], 0, 0, 0);
#pragma unroll
      for (int b = 0; b < CN; ++b) sum[g][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.a[g][1], now.b[b][0], sum[g][b], 0, 0, 0);
#pragma unroll
      for (int b = 0; b < CN; ++b) sum[g][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.a[g][0], now.b[b][0], sum[g][b], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    asked_one();
    slot = next;
  };
  uint32_t k = 0;
  for (; k + 2 <= p.stages; k += 2) {
    stage(even, odd);
    stage(odd, even);
  }
  if (k < p.stages) stage(even, odd);
  wait_and_meet<0>();  // (the loads that found nothing are done, and LDS is read everywhere)

  // A lane has four results of consecutive r for one c.
  const uint32_t r_in = r0 + wr * RN * 16 + lane / 16 * 4, c_in = c0 + wc * CN * 16 + i;
  if (END == kLast) {
#pragma unroll
    for (int a = 0; a < RN; ++a)
#pragma unroll
      for (int b = 0; b < CN; ++b) {
        const uint32_t r = r_in + a * 16, c = c_in + b * 16;
        if (r >= p.rows || c >= p.cols) continue;
        float v[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = sum[a][b][n] * p.scale;
        store_n_within<T, 4>(static_cast<T*>(p.y.p) + plane * p.y.pitch + c * p.y.ld + r, p.rows - r, v);
      }
    return;
  }
  const uint32_t end_r = (p.rows + kBlockCols - 1) / kBlockCols * kBlockCols, end_c = (p.cols + kBlockCols - 1) / kBlockCols * kBlockCols;
  const bool both = !kHalf || place.r != place.c;
  uint32_t* turn = reinterpret_cast<uint32_t*>(lds + wave * K::kTurnBytes);
#pragma unroll
  for (int half = 0; half < RN; half += 2) {
#pragma unroll
    for (int a = half; a < half + 2; ++a)
#pragma unroll
      for (int b = 0; b < CN; ++b) {
        const uint32_t r = r_in + a * 16, c = c_in + b * 16;
        const bool in = c < p.cols && r < end_r;
        v4h high, low;
        float v[4];
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
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          f16_t h, l;
          split(r + n < p.rows && c < p.cols ? v[n] : 0.f, h, l);
          high[n] = h;
          low[n] = l;
          if (both)
            turn[((a - half) * 16 + lane / 16 * 4 + n) * K::kTurnPitch + b * 16 + i] =
                (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
        }
        if (in) {
          char* at = p.by_c.p + plane * p.by_c.pitch + c * p.by_c.ld + pair_at(r);
          *reinterpret_cast<v4h*>(at) = high;
          *reinterpret_cast<v4h*>(at + 64) = low;
        }
      }
    if (!both) continue;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wavefront's own: what its lanes have written is there)
    constexpr uint32_t kEights = CN * 2;  // of a row
#pragma unroll
    for (uint32_t piece = 0; piece < 32 * kEights; piece += kWave) {
      const uint32_t row = (piece + lane) / kEights, eight = (piece + lane) % kEights;
      const uint32_t r = r0 + (wr * RN + half) * 16 + row, c = c0 + wc * CN * 16 + eight * 8;
      const uint32_t* from = turn + row * K::kTurnPitch + eight * 8;
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
}

template <typename T, int END>
void product(const PairTask& p, hipStream_t s) {
  constexpr bool half = END == kGram || END == kPoly;
  auto launch = [&](auto kernel, uint32_t tile, uint32_t threads) {
    kernel<<<dim3(tiles_of(half, (p.rows + tile - 1) / tile, (p.cols + tile - 1) / tile) * p.planes), threads, 0, s>>>(p);
  };
  // tiles of 128 x 128 where there is one for every CU at least
  if ((uint64_t)tiles_of(half, (p.rows + 127) / 128, (p.cols + 127) / 128) * p.planes >= 256)
    launch(pair_kernel<T, END, 4, 4, 2, 2, 2>, 128, 256);
  else
    launch(pair_kernel<T, END, 2, 2, 2, 2, 4>, 64, 256);
}

struct Layout {
  uint64_t n, m;
  bool tall;
  uint32_t parts;
  Pairs x_by_n, x_by_m[2], gram, poly;
  double* part;
  uint64_t bytes;
};

Layout layout_of(const Extent& e, char* scratch) {
  Layout l{};
  l.tall = e.rows > e.cols;
  l.n = std::min(e.rows, e.cols);
  l.m = std::max(e.rows, e.cols);
  const uint64_t elements = e.rows * e.cols;
  l.parts = (uint32_t)std::min<uint64_t>(std::max<uint64_t>(1, 1024 / e.workers), (elements + 8191) / 8192);
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
  return l;
}

template <typename T>
void start(const StartTask& p, uint32_t workers, hipStream_t s) {
  squares_kernel<T><<<dim3(p.parts, workers), kBlock, 0, s>>>(p);
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

size_t orthogonal_bytes(const Extent& e) { return layout_of(e, nullptr).bytes; }

hipError_t launch_orthogonalize(tng_type of_x, tng_type of_y, const Extent& e, const View& x, const float* coefficients, uint32_t steps, float eps, float scale,
                                const View& y, char* scratch, hipStream_t s) {
  const Layout l = layout_of(e, scratch);
  const StartTask first{e.rows, e.cols, x, l.part, l.parts, eps, l.tall, l.x_by_n, l.x_by_m[0]};
  switch (of_x) {
    case TNG_TYPE_F32: start<float>(first, e.workers, s); break;
    case TNG_TYPE_BF16: start<bf16_t>(first, e.workers, s); break;
    default: start<f16_t>(first, e.workers, s); break;
  }
  const uint32_t n = (uint32_t)l.n, m = (uint32_t)l.m, n_stages = (n + kBlockCols - 1) / kBlockCols, m_stages = (m + kBlockCols - 1) / kBlockCols;
  for (uint32_t k = 0; k < steps; ++k) {
    const Pairs &now = l.x_by_m[k % 2], &then = l.x_by_m[1 - k % 2];
    PairTask gram{};
    gram.rows = gram.cols = n;
    gram.stages = m_stages;
    gram.planes = e.workers;
    gram.a = gram.b = l.x_by_n;
    gram.by_r = gram.by_c = l.gram;
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
    apply.scale = scale * (1.f / (kOfPoly * kOfX));
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
