// Dropout from the counter-based generator, and the coders of 8-bit products (gfx950).
#include "tng_layer_device.hpp"

#include <type_traits>

namespace tng {
namespace {

constexpr int kDropout = 0, kResidual = 1, kGrad = 2, kGradRelu = 3;

template <int KIND>
__device__ __forceinline__ float dropout_value(float x, float other, bool keep, const DropArgs& d) {
  if (KIND == kDropout || KIND == kResidual) {
    const float f = (d.relu ? relu(x) : x) * d.scale;
    const float y = keep ? f : 0.f;
    return KIND == kResidual ? other + y : y;
  }
  const bool pass = KIND == kGradRelu ? keep && !(other <= 0.f) : keep;  // (x: the gradient, other: what relu was taken of)
  return pass ? x * d.scale : 0.f;
}

// 16 bytes of a run; STREAM: past the caches.
template <typename T, int N, bool STREAM>
__device__ __forceinline__ void run_in(const T* p, float (&x)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(alignof(T))));
  const GlobalPtr<vec> q = reinterpret_cast<GlobalPtr<vec>>((GlobalPtr<T>)p);
  const vec v = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}
template <typename T, int N, bool STREAM>
__device__ __forceinline__ void run_out(T* p, const float (&x)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(alignof(T))));
  vec v;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (T)x[i];
  if (STREAM)
    __builtin_nontemporal_store(v, reinterpret_cast<vec*>(p));
  else
    *reinterpret_cast<vec*>(p) = v;
}

template <typename T, int KIND, bool STREAM, bool WHOLE>
__device__ __forceinline__ void dropout_piece(uint64_t e, uint64_t n, uint32_t m, const DropArgs& d, const View& x, const View& other,
                                              const View& y) {
  constexpr int N = 16 / sizeof(T);
  constexpr bool kTwo = KIND == kResidual || KIND == kGradRelu;
  const T* from = static_cast<const T*>(x.p) + m * x.pitch + e;
  const T* from_other = static_cast<const T*>(other.p) + (kTwo ? m * other.pitch + e : 0);
  float a[N], b[N];
  if (WHOLE) {  // (no load is under a condition)
    run_in<T, N, STREAM>(from, a);
    if (kTwo) run_in<T, N, STREAM>(from_other, b);
  } else {
    load_n_within<T, N>(from, n - e, 0.f, a);
    if (kTwo) load_n_within<T, N>(from_other, n - e, 0.f, b);
  }
  uint32_t word[N];
  if (d.threshold != 0u) {
    draw_n<N>(e, true, m, d, word);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) word[i] = 0u;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) a[i] = dropout_value<KIND>(a[i], b[i], kept(word[i], d), d);
  T* to = static_cast<T*>(y.p) + m * y.pitch + e;
  if (WHOLE)
    run_out<T, N, STREAM>(to, a);
  else
    store_n_within<T, N>(to, n - e, a);
}

// Rows without gaps: a worker's elements are one run.  A lane takes 16 bytes of each operand; the two blocks of draws that 8
// elements need (50 integer instructions a block) hide under the 48 bytes that they move.  The memory bounds it: 8 x 2048 x 4096
// bfloat16 with a residual, 403 MB, 62.4 us (6.5 TB/s; a fill reaches 6.9, a copy 4.9).
template <typename T, int KIND, bool STREAM>
__global__ void __launch_bounds__(kBlock) dropout_run_kernel(uint64_t n, DropArgs d, View x, View other, View y) {
  constexpr int N = 16 / sizeof(T);
  const uint64_t first = (uint64_t)blockIdx.x * (kBlock * N), e = first + threadIdx.x * N;
  if (first + kBlock * N <= n)
    dropout_piece<T, KIND, STREAM, true>(e, n, blockIdx.y, d, x, other, y);
  else if (e < n)
    dropout_piece<T, KIND, STREAM, false>(e, n, blockIdx.y, d, x, other, y);
}

// Rows with gaps, or of differing pitches: a lane takes one block of four draws, its elements at once where
// they lie in one row: 4 x 2048 x 4000 bfloat16, 131 MB, 34 us (47 one by one).
template <typename T, int KIND>
__global__ void __launch_bounds__(kBlock) dropout_rows_kernel(uint64_t rows, uint64_t cols, DropArgs d, View x, View other, View y) {
  const uint32_t m = blockIdx.y;
  const uint64_t block = (uint64_t)blockIdx.x * kBlock + threadIdx.x, n = rows * cols;
  uint64_t e = block * 4;
  if (e >= n) return;
  uint32_t word[4] = {0u, 0u, 0u, 0u};
  if (d.threshold != 0u) draw_n<4>(e, true, m, d, word);
  uint64_t r = n >> 32 == 0 ? (uint32_t)e / (uint32_t)cols : e / cols, c = e - r * cols;  // (64 bits take four times the instructions)
  constexpr bool kTwo = KIND == kResidual || KIND == kGradRelu;
  if (c + 4 <= cols) {  // (all four of one row)
    float a[4], b[4];
    load_n<T, 4>(static_cast<const T*>(x.p) + m * x.pitch + r * x.ld + c, a);
    if (kTwo) load_n<T, 4>(static_cast<const T*>(other.p) + m * other.pitch + r * other.ld + c, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = dropout_value<KIND>(a[i], b[i], kept(word[i], d), d);
    store_n_within<T, 4>(static_cast<T*>(y.p) + m * y.pitch + r * y.ld + c, 4, a);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (e + i < n) {
      const float a = (float)static_cast<const T*>(x.p)[m * x.pitch + r * x.ld + c];
      float b = 0.f;
      if (kTwo) b = (float)static_cast<const T*>(other.p)[m * other.pitch + r * other.ld + c];
      static_cast<T*>(y.p)[m * y.pitch + r * y.ld + c] = (T)dropout_value<KIND>(a, b, kept(word[i], d), d);
    }
    if (++c == cols) {
      c = 0;
      ++r;
    }
  }
}

template <typename T, int KIND>
hipError_t dropout_typed(const Extent& n, const DropArgs& d, const View& x, const View& other, const View& y, hipStream_t s) {
  const uint64_t elements = n.rows * n.cols;
  const bool two = KIND == kResidual || KIND == kGradRelu;
  const bool run = n.rows == 1 || (x.ld == n.cols && y.ld == n.cols && (!two || other.ld == n.cols));
  const uint64_t per = run ? kBlock * (16 / sizeof(T)) : kBlock * 4;
  const dim3 grid((uint32_t)((elements + per - 1) / per), n.workers);
  // Past the caches where the operands together are more than the memory-side cache holds; of less, what comes next finds y in there.  Both sides, us,
  // past / through the caches, bfloat16, the call alone and with the coder of y's rows behind it: with a residual 32 MiB each 16.2 / 16.9 and
  // 29.7 / 26.5, 80 MiB 38.9 / 36.7 and 63.4 / 59.9, 96 MiB 46.9 / 52.5 and 75.9 / 73.6, 128 MiB 60.2 / 67.5 and 96.3 / 98.9; without one 128 MiB 42.3 /
  // 41.8 and 76.0 / 73.2, 192 MiB 66.2 / 67.4 and 109.4 / 121.5.
  const uint64_t bytes = elements * n.workers * sizeof(T) * (two ? 3 : 2);
  if (run && bytes > (256u << 20))
    dropout_run_kernel<T, KIND, true><<<grid, kBlock, 0, s>>>(elements, d, x, other, y);
  else if (run)
    dropout_run_kernel<T, KIND, false><<<grid, kBlock, 0, s>>>(elements, d, x, other, y);
  else
    dropout_rows_kernel<T, KIND><<<grid, kBlock, 0, s>>>(n.rows, n.cols, d, x, other, y);
  return hipGetLastError();
}

template <int KIND>
hipError_t dropout_kind(tng_type type, const Extent& n, const DropArgs& d, const View& x, const View& other, const View& y,
                        hipStream_t s) {
  switch (type) {
    case TNG_TYPE_F32: return dropout_typed<float, KIND>(n, d, x, other, y, s);
    case TNG_TYPE_BF16: return dropout_typed<bf16_t, KIND>(n, d, x, other, y, s);
    default: return dropout_typed<f16_t, KIND>(n, d, x, other, y, s);
  }
}

// ---- codes of rows

// A lane takes eight columns.  Where a row ends inside them it takes the row's last eight instead: what two lanes have of one column is the
// same, and so is what they write there.  No load is under a condition, so many are under way together (a load that only some lanes
// make is waited for where the ways join again).  NARROW: rows of less than eight columns.
template <bool NARROW>
__device__ __forceinline__ uint64_t eight_at(uint64_t c, uint64_t cols) {
  return NARROW ? c : min(c, cols - 8);
}

template <typename T, bool NARROW>
__device__ __forceinline__ void load8(const T* row, uint64_t c, uint64_t cols, float (&v)[8]) {
  if (NARROW)
    load_n_within<T, 8>(row + c, c < cols ? cols - c : 0, 0.f, v);
  else
    load_n<T, 8>(row + c, v);
}

// The same as they lie, for loads that are under way while something else is worked on.
template <typename T, bool NARROW>
struct Raw8 {
  typedef T vec __attribute__((ext_vector_type(8), aligned(alignof(T))));
  vec v;
  __device__ __forceinline__ void load(const T* row, uint64_t c, uint64_t cols) {
    if (NARROW) {
      for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? row[c + i] : (T)0.f;
    } else {
      v = *reinterpret_cast<GlobalPtr<vec>>((GlobalPtr<T>)(row + c));
    }
  }
};

template <bool NARROW>
__device__ __forceinline__ void store_codes8(int8_t* p, uint64_t count, const uint32_t (&q)[8]) {
  typedef uint32_t two __attribute__((ext_vector_type(2), aligned(1)));
  two v;
  v.x = pack4(q[0], q[1], q[2], q[3]);
  v.y = pack4(q[4], q[5], q[6], q[7]);
  if (!NARROW) {
    *reinterpret_cast<two*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((uint64_t)i < count) p[i] = (int8_t)(v[i / 4] >> (i % 4 * 8));
  }
}

// What drop makes of columns c .. c + 7 of a row whose first element is number `first`.
__device__ __forceinline__ void drop_values(float (&v)[8], uint64_t c, uint64_t cols, uint64_t first, uint32_t m, const DropArgs& d) {
  uint32_t word[8];
  if (d.threshold != 0u) {
    draw_n<8>(first + c, (cols & 3u) == 0u, m, d, word);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) word[i] = 0u;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = dropped(v[i], word[i], d);
}

// LANES take one row, and hold it: HELD times 8 columns each.  A wavefront needs no barrier, a workgroup has a long row sooner.  One read of
// the row and one write of its codes bound it: 8192 x 2048 bfloat16, 50 MB, 10 us (5 TB/s); with dropout 14, by the draws' instructions.
template <typename T, bool DROP, int LANES, int HELD, bool NARROW>
__global__ void __launch_bounds__(kBlock) quantize_rows_kernel(uint64_t all, uint64_t rows, uint64_t cols, DropArgs d, View x, View q,
                                                               float* scale) {
  const uint32_t lane = threadIdx.x % LANES;
  const uint64_t index = (uint64_t)blockIdx.x * (kBlock / LANES) + __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
  if (LANES == kWave && index >= all) return;  // (one row for a workgroup: none is left over)
  const uint32_t m = (uint32_t)index / (uint32_t)rows;
  const uint64_t r = index - m * rows;
  const T* row = static_cast<const T*>(x.p) + m * x.pitch + r * x.ld;
  int8_t* out = static_cast<int8_t*>(q.p) + m * q.pitch + r * q.ld;
  float v[HELD][8];
  uint32_t top = 0u;
#pragma unroll
  for (int k = 0; k < HELD; ++k) load8<T, NARROW>(row, eight_at<NARROW>((k * LANES + lane) * 8, cols), cols, v[k]);
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    if (DROP) drop_values(v[k], eight_at<NARROW>((k * LANES + lane) * 8, cols), cols, r * cols, m, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(v[k][i]));
  }
  top = wave_max_bits(top);
  if (LANES > kWave) {
    __shared__ uint32_t tops[kBlock / kWave];
    if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kBlock / kWave; ++k) top = max(top, tops[k]);
  }
  const float inv = code_inverse(top);
  if (lane == 0) scale[index] = code_step(top);
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    const uint64_t c = (k * LANES + lane) * 8;
    uint32_t code[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) code[i] = code_nearest(v[k][i], inv);
    if (c < cols) store_codes8<NARROW>(out + eight_at<NARROW>(c, cols), cols - c, code);
  }
}

// Longer rows, a workgroup each: read (and drawn) again for the codes, mostly from a cache (4096 x 20000 bfloat16, 246 MB, 59 us).
template <typename T, bool DROP>
__global__ void __launch_bounds__(kBlock) quantize_long_rows_kernel(uint64_t rows, uint64_t cols, DropArgs d, View x, View q, float* scale) {
  const uint64_t index = blockIdx.x;
  const uint32_t m = (uint32_t)index / (uint32_t)rows;
  const uint64_t r = index - m * rows;
  const T* row = static_cast<const T*>(x.p) + m * x.pitch + r * x.ld;
  int8_t* out = static_cast<int8_t*>(q.p) + m * q.pitch + r * q.ld;
  float v[8];
  uint32_t top = 0u;
#pragma unroll 4
  for (uint64_t c = threadIdx.x * 8; c < cols; c += kBlock * 8) {
    const uint64_t at = eight_at<false>(c, cols);
    load8<T, false>(row, at, cols, v);
    if (DROP) drop_values(v, at, cols, r * cols, m, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(v[i]));
  }
  __shared__ uint32_t tops[kBlock / kWave];
  top = wave_max_bits(top);
  if (threadIdx.x % kWave == 0) tops[threadIdx.x / kWave] = top;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kBlock / kWave; ++k) top = max(top, tops[k]);
  const float inv = code_inverse(top);
  if (threadIdx.x == 0) scale[index] = code_step(top);
#pragma unroll 2
  for (uint64_t c = threadIdx.x * 8; c < cols; c += kBlock * 8) {
    const uint64_t at = eight_at<false>(c, cols);
    uint32_t code[8];
    load8<T, false>(row, at, cols, v);
    if (DROP) drop_values(v, at, cols, r * cols, m, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) code[i] = code_nearest(v[i], inv);
    store_codes8<false>(out + at, 8, code);
  }
}

// Few rows get a workgroup each, for their latency, many a wavefront each.  (Both, us: 1 row of 4096 bfloat16 2.5 / 4; 8192 rows of 2048 with
// dropout, in the midst of a step, 27 / 19.)
template <typename T, bool DROP>
void quantize_rows_typed(const Extent& n, const DropArgs& d, const View& x, const View& q, float* scale, hipStream_t s) {
  const uint64_t all = n.workers * n.rows;
  auto launch = [&](auto lanes, auto held, auto narrow) {
    constexpr int each = kBlock / lanes;
    quantize_rows_kernel<T, DROP, lanes, held, narrow>
        <<<dim3((uint32_t)((all + each - 1) / each)), kBlock, 0, s>>>(all, n.rows, n.cols, d, x, q, scale);
  };
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  constexpr std::integral_constant<int, 4> four;
  constexpr std::integral_constant<int, 8> eight;
  constexpr std::integral_constant<int, kWave> wave;
  constexpr std::integral_constant<int, kBlock> block;
  if (n.cols < 8)
    launch(wave, one, std::true_type{});
  else if (n.cols <= 512)
    launch(wave, one, std::false_type{});
  else if (all >= 1024 && n.cols <= 1024)
    launch(wave, two, std::false_type{});
  else if (all >= 1024 && n.cols <= 2048)
    launch(wave, four, std::false_type{});
  else if (all >= 1024 && n.cols <= 4096)
    launch(wave, eight, std::false_type{});
  else if (n.cols <= 2048)
    launch(block, one, std::false_type{});
  else if (n.cols <= 4096)
    launch(block, two, std::false_type{});
  else if (n.cols <= 8192)
    launch(block, four, std::false_type{});
  else
    quantize_long_rows_kernel<T, DROP><<<dim3((uint32_t)all), kBlock, 0, s>>>(n.rows, n.cols, d, x, q, scale);
}

// ---- codes the other way round.  A tile is ROWS x 128 codes; in LDS they lie as [column][row], 16-byte pieces of a column's rows moved
// by the column's number / 16 so that the writes of a wavefront do not meet in one bank.
constexpr int kTile = 128;

template <int ROWS>
__device__ __forceinline__ uint32_t turned_at(uint32_t col, uint32_t group) {  // 4-byte word of rows 4 group .. 4 group + 3
  return col * (ROWS / 4) + (group ^ ((col >> 4 << 2) & (ROWS / 4 - 1)));
}

// words: [kTile][ROWS / 4].  Columns c0 .. of a worker's matrix become rows of qt, r0 .. its columns.
template <int ROWS>
__device__ __forceinline__ void store_turned(const uint32_t* words, const View& qt, uint32_t m, uint64_t r0, uint64_t c0, uint64_t rows,
                                             uint64_t cols) {
  typedef uint32_t four __attribute__((ext_vector_type(4)));
  typedef uint32_t four_any __attribute__((ext_vector_type(4), aligned(1)));
#pragma unroll
  for (int k = 0; k < kTile * ROWS / 16 / kBlock; ++k) {
    const uint32_t piece = k * kBlock + threadIdx.x, col = piece / (ROWS / 16), at = piece % (ROWS / 16);
    const uint64_t r = r0 + at * 16;
    if (c0 + col >= cols || r >= rows) continue;
    const four v = *reinterpret_cast<const four*>(words + turned_at<ROWS>(col, at * 4));
    int8_t* p = static_cast<int8_t*>(qt.p) + m * qt.pitch + (c0 + col) * qt.ld + r;
    if (rows - r >= 16) {
      *reinterpret_cast<four_any*>(p) = v;
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 16; ++i)
        if (i < rows - r) p[i] = (int8_t)(v[i / 4] >> (i % 4 * 8));
    }
  }
}

// Four words of four codes each, turned: byte k of word i becomes byte i of word k.
__device__ __forceinline__ void turn4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), e = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(e, b, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(e, b, 0x07060302u);
}

// 8192 x 2048 codes, 34 MB, 6.8 us; few tiles take the latency of their one load and one store, 4 to 5.
__global__ void __launch_bounds__(kBlock) turn_codes_kernel(uint64_t rows, uint64_t cols, View q, View qt) {
  __shared__ __align__(16) uint32_t words[kTile * kTile / 4];
  const uint32_t m = blockIdx.z, chunk = threadIdx.x % 8, group = threadIdx.x / 8;
  const uint64_t r0 = (uint64_t)blockIdx.y * kTile, c0 = (uint64_t)blockIdx.x * kTile;
  // 16 columns a lane; the last 16 where a row ends inside them (as eight_at)
  const bool narrow = cols < 16, some = c0 + chunk * 16 < cols;
  const uint64_t c = narrow ? c0 + chunk * 16 : min(c0 + chunk * 16, cols - 16);
  const int at = narrow ? (int)chunk * 16 : (int)((int64_t)c - (int64_t)c0);
  typedef uint32_t four __attribute__((ext_vector_type(4), aligned(1)));
  four w[4];
  if (!narrow) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = *reinterpret_cast<const four*>(static_cast<const int8_t*>(q.p) + m * q.pitch + min(r0 + group * 4 + i, rows - 1) * q.ld + c);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int8_t* p = static_cast<const int8_t*>(q.p) + m * q.pitch + min(r0 + group * 4 + i, rows - 1) * q.ld + c;
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) w[i][k] = 0u;
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k)
        if (c + k < cols) w[i][k / 4] |= (uint32_t)(uint8_t)p[k] << (k % 4 * 8);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t t[4] = {w[0][k], w[1][k], w[2][k], w[3][k]};
    turn4(t);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (some && at + k * 4 + j >= 0) words[turned_at<kTile>(at + k * 4 + j, group)] = t[j];
  }
  __syncthreads();
  store_turned<kTile>(words, qt, m, r0, c0, rows, cols);
}

// ---- codes of a gradient
//
// dy[t][n] is coded twice: dy[t][n] col_scale[n] along n (one scale a row, for the product with the weights' codes) and
// dy[t][n] row_scale[t] along t (one scale a column of a worker, for the product with the tokens' codes).  The first kernel takes
// both kinds of maxima and the columns' sums in one pass, the second puts the pieces together, the third codes.  4 x 2048 x 8192 bfloat16: all
// 96 us; the first 27, its 134 MB at 5 TB/s (56 in a step, where the result of a product is still on its way to the memory), the second 5, the
// third 67, by the vector instructions: 40 for an element, of which the draws are 12.
constexpr int kStatCols = kWave * 8;

// Rows of a chunk: a wavefront takes a quarter of them, one pair after another, so few where that still leaves every CU a workgroup.
uint32_t chunk_rows(const Extent& n) {
  const uint64_t tiles = (n.cols + kStatCols - 1) / kStatCols;
  for (const uint32_t rows : {64u, 32u, 16u})
    if (n.workers * tiles * ((n.rows + rows - 1) / rows) >= 512) return rows;
  return 8u;
}

struct GradScratch {
  float *row_inv, *col_inv;         // [workers][rows], [workers][cols]
  uint32_t *row_part, *col_part;    // [workers][column tiles][rows], [workers][row chunks][cols]
  float* sum_part;                  // [workers][row chunks][cols]
};

template <typename T, bool NARROW>
__global__ void __launch_bounds__(kBlock) grad_stats_kernel(uint64_t rows, uint64_t cols, uint32_t tiles, uint32_t chunks, uint32_t each, View dy,
                                                            const float* col_scale, const float* row_scale, GradScratch out) {
  constexpr int kWaves = kBlock / kWave, kMany = 2;  // rows at a time, and as many under way
  const uint32_t m = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t chunk = blockIdx.x / tiles, tile = blockIdx.x - chunk * tiles;
  const uint64_t c0 = (uint64_t)tile * kStatCols, c = eight_at<NARROW>(c0 + lane * 8, cols);
  const uint64_t r0 = (uint64_t)chunk * each + wave * (each / kWaves);
  const uint64_t end = min(rows, r0 + each / kWaves);
  float scale[8], sum[8];
  uint32_t top[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    scale[i] = 1.f;
    sum[i] = 0.f;
    top[i] = 0u;
  }
  if (col_scale != nullptr) load8<float, NARROW>(col_scale, c, cols, scale);
  Raw8<T, NARROW> raw[kMany], coming[kMany];
  float s[kMany], coming_s[kMany];
  auto ask = [&](uint64_t r, Raw8<T, NARROW>(&x)[kMany], float (&f)[kMany]) {
#pragma unroll
    for (int k = 0; k < kMany; ++k) {  // (past the end: the last row again, which is not counted)
      const uint64_t row = min(r + k, rows - 1);
      x[k].load(static_cast<const T*>(dy.p) + m * dy.pitch + row * dy.ld, c, cols);
      f[k] = row_scale != nullptr ? row_scale[m * rows + row] : 1.f;
    }
  };
  ask(r0, raw, s);
#pragma unroll 1
  for (uint64_t r = r0; r < end; r += kMany) {
    ask(r + kMany, coming, coming_s);
    uint32_t t[kMany];
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      const bool in = r + k < end;
      t[k] = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = (float)raw[k].v[i];
        t[k] = max(t[k], magnitude_bits(v * scale[i]));
        top[i] = max(top[i], magnitude_bits(v * s[k]));
        sum[i] += in ? v : 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      t[k] = wave_max_bits(t[k]);
      if (lane == 0 && r + k < end) out.row_part[((uint64_t)m * tiles + tile) * rows + r + k] = t[k];
    }
#pragma unroll
    for (int k = 0; k < kMany; ++k) {
      raw[k] = coming[k];
      s[k] = coming_s[k];
    }
  }
  __shared__ uint32_t tops[kWaves][kStatCols];
  __shared__ float sums[kWaves][kStatCols];
  const int at = NARROW ? (int)lane * 8 : (int)((int64_t)c - (int64_t)c0);  // (before the tile, in a last tile of less than eight columns)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (at + i >= 0) {
      tops[wave][at + i] = top[i];
      sums[wave][at + i] = sum[i];
    }
  }
  __syncthreads();
  for (uint32_t j = threadIdx.x; j < kStatCols; j += kBlock) {
    const uint64_t n = (uint64_t)tile * kStatCols + j;
    if (n >= cols) break;
    uint32_t t = 0u;
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      t = max(t, tops[w][j]);
      a += sums[w][j];
    }
    const uint64_t at = ((uint64_t)m * chunks + chunk) * cols + n;
    out.col_part[at] = t;
    out.sum_part[at] = a;
  }
}

// The maximum (and the sum) of n partial results that are `stride` apart, MANY under way at a time.
template <uint32_t MANY, typename Offset>
__device__ __forceinline__ uint32_t max_of(const uint32_t* p, uint32_t n, Offset stride) {
  uint32_t top = 0u;
  for (uint32_t k = 0; k < n; k += MANY) {
    uint32_t t[MANY];
#pragma unroll
    for (uint32_t i = 0; i < MANY; ++i) t[i] = p[min(k + i, n - 1) * stride];
#pragma unroll
    for (uint32_t i = 0; i < MANY; ++i) top = max(top, t[i]);
  }
  return top;
}
template <uint32_t MANY, typename Offset>
__device__ __forceinline__ float sum_of(const float* p, uint32_t n, Offset stride) {
  float sum = 0.f;
  for (uint32_t k = 0; k < n; k += MANY) {
    float t[MANY];
#pragma unroll
    for (uint32_t i = 0; i < MANY; ++i) t[i] = p[min(k + i, n - 1) * stride];
#pragma unroll
    for (uint32_t i = 0; i < MANY; ++i) sum += k + i < n ? t[i] : 0.f;
  }
  return sum;
}

// What the statistics' pieces go to: where a product reads the scales, and the columns' sums (may be null).
struct GradResults {
  float *q_scale, *qt_scale, *col_sum;
};

// Row r and column c of worker m: its scale (and sum) out, the inverse of its largest magnitude back.
__device__ __forceinline__ float finish_row(const GradScratch& in, const GradResults& out, uint32_t m, uint64_t r, uint64_t rows, uint32_t tiles,
                                            bool write) {
  const uint32_t top = max_of<8>(in.row_part + (uint64_t)m * tiles * rows + r, tiles, rows);
  if (write) out.q_scale[m * rows + r] = code_step(top);
  return code_inverse(top);
}
template <uint32_t MANY, typename Offset>
__device__ __forceinline__ float finish_col(const GradScratch& in, const GradResults& out, uint32_t m, uint64_t c, uint64_t cols,
                                            uint32_t chunks, bool write) {
  const uint64_t at = (uint64_t)m * chunks * cols + c;
  const uint32_t top = max_of<MANY>(in.col_part + at, chunks, (Offset)cols);
  if (write) {
    out.qt_scale[m * cols + c] = code_step(top);
    if (out.col_sum != nullptr) out.col_sum[m * cols + c] = sum_of<MANY>(in.sum_part + at, chunks, (Offset)cols);
  }
  return code_inverse(top);
}

// One lane a row or a column: rows first (blockIdx.x < row_blocks), then columns.
__global__ void __launch_bounds__(kBlock) grad_finish_kernel(uint64_t rows, uint64_t cols, uint32_t tiles, uint32_t chunks,
                                                             uint32_t row_blocks, GradScratch in, GradResults out) {
  const uint32_t m = blockIdx.y;
  const bool by_rows = blockIdx.x < row_blocks;
  const uint64_t j = (uint64_t)(by_rows ? blockIdx.x : blockIdx.x - row_blocks) * kBlock + threadIdx.x;
  if (by_rows) {
    if (j < rows) in.row_inv[m * rows + j] = finish_row(in, out, m, j, rows, tiles, true);
  } else {
    if (j < cols) in.col_inv[m * cols + j] = finish_col<8, uint64_t>(in, out, m, j, cols, chunks, true);
  }
}

// HALVES times 64 rows for a workgroup: one where there are few tiles, for its time.  JOINS: it puts the statistics of its rows and columns
// together itself, where that is less than a launch.
template <typename T, bool NARROW, int HALVES, bool JOINS>
__global__ void __launch_bounds__(kBlock, 4) grad_codes_kernel(uint64_t rows, uint64_t cols, DropArgs key, View dy, const float* col_scale,
                                                            const float* row_scale, GradScratch in, GradResults out, uint32_t tiles,
                                                            uint32_t chunks, View q, View qt) {
  constexpr int kRows = HALVES * 64;
  static_assert(!JOINS || HALVES == 1, "what it asks for first is all that it reads");
  __shared__ __align__(16) uint32_t words[kTile * kRows / 4];
  const uint32_t m = blockIdx.z, chunk = threadIdx.x % 16, group = threadIdx.x / 16;
  const uint64_t r0 = (uint64_t)blockIdx.y * kRows, c0 = (uint64_t)blockIdx.x * kTile, c = eight_at<NARROW>(c0 + chunk * 8, cols);
  const bool some = c0 + chunk * 8 < cols;
  const int at = NARROW ? (int)chunk * 8 : (int)((int64_t)c - (int64_t)c0);  // (before the tile, in a last tile of less than eight columns)
  float scale[8], inv[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) scale[i] = 1.f;
  if (col_scale != nullptr) load8<float, NARROW>(col_scale, c, cols, scale);
  Raw8<T, NARROW> raw[4];
  float s[4];
  auto ask = [&](uint64_t r) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // (past the end: the last row again, whose codes go nowhere)
      const uint64_t row = min(r + k, rows - 1);
      raw[k].load(static_cast<const T*>(dy.p) + m * dy.pitch + row * dy.ld, c, cols);
      s[k] = row_scale != nullptr ? row_scale[m * rows + row] : 1.f;
    }
  };
  __shared__ float row_invs[JOINS ? kRows : 1], col_invs[JOINS ? kTile : 1];
  if (JOINS) {
    ask(r0 + group * 4);  // (under way while the pieces are put together, sixteen at a time: 8 x 512 x 1024 float16 13.4 -> 12.3 us)
    const uint32_t j = threadIdx.x % kTile;
    if (threadIdx.x < kTile) {
      if (j < kRows && r0 + j < rows) row_invs[j] = finish_row(in, out, m, r0 + j, rows, tiles, blockIdx.x == 0);
    } else if (c0 + j < cols) {
      col_invs[j] = finish_col<16, uint32_t>(in, out, m, c0 + j, cols, chunks, blockIdx.y == 0);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = col_invs[min(max(at + i, 0), kTile - 1)];
  } else {
    load8<float, NARROW>(in.col_inv + m * cols, c, cols, inv);
  }
#pragma unroll 1
  for (uint32_t half = 0; half < HALVES; ++half) {
    const uint32_t g = group + half * 16;
    const uint64_t r = r0 + g * 4;
    if (!JOINS) ask(r);
    float row_inv[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint64_t row = min(r + k, rows - 1);
      row_inv[k] = JOINS ? row_invs[row - r0] : in.row_inv[m * rows + row];
    }
    uint32_t down[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t word[8], code[8];
      draw_n<8>((r + k) * cols + c, (cols & 3u) == 0u, m, key, word);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = (float)raw[k].v[i];
        code[i] = code_drawn(v * scale[i], row_inv[k], word[i] >> 16);
        down[k][i] = code_drawn(v * s[k], inv[i], word[i] & 0xFFFFu);
      }
      if (some && r + k < rows) store_codes8<NARROW>(static_cast<int8_t*>(q.p) + m * q.pitch + (r + k) * q.ld + c, cols - c, code);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i >= 0 && some) words[turned_at<kRows>(at + i, g)] = pack4(down[0][i], down[1][i], down[2][i], down[3][i]);
  }
  __syncthreads();
  store_turned<kRows>(words, qt, m, r0, c0, rows, cols);
}

GradScratch grad_scratch(const Extent& n, float* p) {
  const uint64_t tiles = (n.cols + kStatCols - 1) / kStatCols, chunks = (n.rows + chunk_rows(n) - 1) / chunk_rows(n);
  GradScratch g;
  g.row_inv = p;
  p += n.workers * n.rows;
  g.col_inv = p;
  p += n.workers * n.cols;
  g.row_part = reinterpret_cast<uint32_t*>(p);
  p += n.workers * tiles * n.rows;
  g.col_part = reinterpret_cast<uint32_t*>(p);
  p += n.workers * chunks * n.cols;
  g.sum_part = p;
  return g;
}

template <typename T, bool NARROW>
hipError_t quantize_grad_typed(const Extent& n, const DropArgs& key, const View& dy, const float* col_scale, const float* row_scale,
                               const View& q, float* q_scale, const View& qt, float* qt_scale, float* col_sum, float* scratch,
                               hipStream_t s) {
  const GradScratch g = grad_scratch(n, scratch);
  const uint32_t each = chunk_rows(n);
  const uint32_t tiles = (uint32_t)((n.cols + kStatCols - 1) / kStatCols), chunks = (uint32_t)((n.rows + each - 1) / each);
  const bool none = n.rows == 0 || n.cols == 0;  // (scales and sums are 0 then)
  if (!none) grad_stats_kernel<T, NARROW><<<dim3(tiles * chunks, n.workers), kBlock, 0, s>>>(n.rows, n.cols, tiles, chunks, each, dy, col_scale, row_scale, g);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const GradResults out{q_scale, qt_scale, col_sum};
  // Which kernel codes, and with it who puts the statistics together: from 1024 whole tiles on workgroups of two halves, whose statistics
  // grad_finish_kernel makes (a step of 4 x 2048 tokens, 8192 channels would read the pieces 4096 times); of fewer, workgroups of one half, that join
  // few pieces themselves (a step of 3 x 111 tokens, 1003 channels 48 -> 45 us).
  enum class Codes { kTwoHalves, kOneHalf, kJoining };
  const uint32_t across = (uint32_t)((n.cols + kTile - 1) / kTile);
  auto down = [&](uint64_t halves) { return (n.rows + halves * 64 - 1) / (halves * 64); };
  Codes codes = Codes::kOneHalf;
  if (down(2) * across * n.workers >= 1024)
    codes = Codes::kTwoHalves;
  else if (!none && down(1) * across * n.workers <= 1024 && tiles <= 32 && chunks <= 64)
    codes = Codes::kJoining;
  if (codes != Codes::kJoining) {
    const uint32_t row_blocks = (uint32_t)((n.rows + kBlock - 1) / kBlock), col_blocks = (uint32_t)((n.cols + kBlock - 1) / kBlock);
    grad_finish_kernel<<<dim3(row_blocks + col_blocks, n.workers), kBlock, 0, s>>>(n.rows, n.cols, tiles, chunks, row_blocks, g, out);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || none) return e;
  }
  auto launch = [&](auto halves, auto joining) {
    grad_codes_kernel<T, NARROW, halves, joining><<<dim3(across, (uint32_t)down(halves), n.workers), kBlock, 0, s>>>(
        n.rows, n.cols, key, dy, col_scale, row_scale, g, out, tiles, chunks, q, qt);
  };
  switch (codes) {
    case Codes::kTwoHalves: launch(std::integral_constant<int, 2>{}, std::false_type{}); break;
    case Codes::kOneHalf: launch(std::integral_constant<int, 1>{}, std::false_type{}); break;
    case Codes::kJoining: launch(std::integral_constant<int, 1>{}, std::true_type{}); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(tng_type type, const Extent& n, const DropArgs& d, const View& x, const View& residual, const View& y,
                          hipStream_t s) {
  return residual.p != nullptr ? dropout_kind<kResidual>(type, n, d, x, residual, y, s) : dropout_kind<kDropout>(type, n, d, x, residual, y, s);
}

hipError_t launch_dropout_grad(tng_type type, const Extent& n, const DropArgs& d, const View& x, const View& dy, const View& dx,
                               hipStream_t s) {
  return d.relu ? dropout_kind<kGradRelu>(type, n, d, dy, x, dx, s) : dropout_kind<kGrad>(type, n, d, dy, x, dx, s);
}

hipError_t launch_quantize_rows(tng_type type, const Extent& n, const DropArgs* drop, const View& x, const View& q, float* scale,
                                const View& qt, hipStream_t s) {
  const DropArgs d = drop != nullptr ? *drop : DropArgs{};
  switch (type) {
    case TNG_TYPE_F32:
      drop ? quantize_rows_typed<float, true>(n, d, x, q, scale, s) : quantize_rows_typed<float, false>(n, d, x, q, scale, s);
      break;
    case TNG_TYPE_BF16:
      drop ? quantize_rows_typed<bf16_t, true>(n, d, x, q, scale, s) : quantize_rows_typed<bf16_t, false>(n, d, x, q, scale, s);
      break;
    default:
      drop ? quantize_rows_typed<f16_t, true>(n, d, x, q, scale, s) : quantize_rows_typed<f16_t, false>(n, d, x, q, scale, s);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess || qt.p == nullptr) return e;
  return launch_turn_codes(n, q, qt, s);
}

hipError_t launch_turn_codes(const Extent& n, const View& q, const View& qt, hipStream_t s) {
  const dim3 grid((uint32_t)((n.cols + kTile - 1) / kTile), (uint32_t)((n.rows + kTile - 1) / kTile), n.workers);
  turn_codes_kernel<<<grid, kBlock, 0, s>>>(n.rows, n.cols, q, qt);
  return hipGetLastError();
}

size_t quantize_grad_floats(const Extent& n) {
  const uint64_t tiles = (n.cols + kStatCols - 1) / kStatCols, chunks = (n.rows + chunk_rows(n) - 1) / chunk_rows(n);
  return n.workers * (n.rows + n.cols + tiles * n.rows + 2 * chunks * n.cols);
}

hipError_t launch_quantize_grad(tng_type type, const Extent& n, const DropArgs& key, const View& dy, const float* col_scale,
                                const float* row_scale, const View& q, float* q_scale, const View& qt, float* qt_scale, float* col_sum,
                                float* scratch, hipStream_t s) {
  auto launch = [&](auto narrow) {
    switch (type) {
      case TNG_TYPE_F32:
        return quantize_grad_typed<float, narrow>(n, key, dy, col_scale, row_scale, q, q_scale, qt, qt_scale, col_sum, scratch, s);
      case TNG_TYPE_BF16:
        return quantize_grad_typed<bf16_t, narrow>(n, key, dy, col_scale, row_scale, q, q_scale, qt, qt_scale, col_sum, scratch, s);
      default:
        return quantize_grad_typed<f16_t, narrow>(n, key, dy, col_scale, row_scale, q, q_scale, qt, qt_scale, col_sum, scratch, s);
    }
  };
  return n.cols < 8 ? launch(std::true_type{}) : launch(std::false_type{});
}

}  // namespace tng
