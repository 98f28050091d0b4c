// Root-mean-square norms: the residual's addition in front, 8-bit codes behind, and the gradient (gfx950).
#include "tng_layer_device.hpp"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace tng {
namespace {

// A lane takes eight columns, and where a row ends inside them the row's last eight, as the coders do.  Here the first `shift` of those are another
// lane's: they count as 0, and are not written.  So no lane needs what another one may have overwritten (results may lie where inputs do).
struct Eight {
  uint32_t at, shift;  // shift 8: nothing is left for this lane
};
template <bool NARROW>
__device__ __forceinline__ Eight eight_of(uint64_t c, uint64_t cols) {
  if (NARROW) return Eight{0, c == 0 ? 0u : 8u};
  const uint32_t at = (uint32_t)min(c, cols - 8);
  return Eight{at, min((uint32_t)c - at, 8u)};
}

template <typename T>
using Vec8 = T __attribute__((ext_vector_type(8), aligned(alignof(T))));

// NARROW: rows of less than eight columns, all of them the first lane's.
template <typename T, bool NARROW>
__device__ __forceinline__ Vec8<T> load_eight(const T* row, const Eight& e, uint64_t cols) {
  Vec8<T> v;
  if (NARROW) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = e.shift == 0 && i < cols ? row[i] : (T)0.f;
  } else {
    v = *reinterpret_cast<GlobalPtr<Vec8<T>>>((GlobalPtr<T>)(row + e.at));
  }
  return v;
}

template <typename T, bool NARROW>
__device__ __forceinline__ void store_eight(T* row, const Eight& e, uint64_t cols, const Vec8<T>& v) {
  if (!NARROW && e.shift == 0) {
    *reinterpret_cast<Vec8<T>*>(row + e.at) = v;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i >= e.shift && (!NARROW || i < cols)) row[e.at + i] = v[i];
  }
}

template <typename T>
__device__ __forceinline__ void widen(const Vec8<T>& v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
template <typename T>
__device__ __forceinline__ Vec8<T> narrowed(const float (&x)[8]) {
  Vec8<T> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
  return v;
}

template <bool NARROW>
__device__ __forceinline__ void load_weight(const float* weight, const Eight& e, uint64_t cols, float (&w)[8]) {
  if (weight != nullptr) {
    widen<float>(load_eight<float, NARROW>(weight, e, cols), w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
  }
}

__device__ __forceinline__ float wave_sum(float x) {
  x = plus_other<0xB1, 0xF>(x);  // the neighbour, the pair, the half and the row of 16
  x = plus_other<0x4E, 0xF>(x);
  x = plus_other<0x141, 0xF>(x);
  x = plus_other<0x140, 0xF>(x);
  x = plus_other<0x142, 0xA>(x);  // rows 0 and 2 into 1 and 3, then 1 into 3
  x = plus_other<0x143, 0xC>(x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Joins over the LANES that share a row.  Every lane of the workgroup comes here as often as the others.
template <int LANES>
struct Joint {
  static constexpr int kWaves = LANES / kWave;
  float (*of_sum)[2];
  uint32_t* of_max;
  uint32_t first, wave;  // the group's first wavefront, and this lane's
  __device__ __forceinline__ void sum(float& a, float& b) const {
    a = wave_sum(a);
    b = wave_sum(b);
    if (kWaves == 1) return;
    __syncthreads();  // (what was joined before has been read)
    if (threadIdx.x % kWave == 0) {
      of_sum[wave][0] = a;
      of_sum[wave][1] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      a += of_sum[first + k][0];
      b += of_sum[first + k][1];
    }
  }
  __device__ __forceinline__ float sum(float a) const {
    float none = 0.f;
    sum(a, none);
    return a;
  }
  __device__ __forceinline__ uint32_t max_bits(uint32_t top) const {
    top = wave_max_bits(top);
    if (kWaves == 1) return top;
    if (threadIdx.x % kWave == 0) of_max[wave] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) top = max(top, of_max[first + k]);
    return top;
  }
};

// 1 / sqrt(mean + eps) from the sum of squares.  squares(f): the sum of (h f)^2, taken again where the squares of large numbers are beyond
// binary32 (eps is nothing beside them).  A row that holds what is not finite is NaN as a whole.
// f = 2^-80: of 2^22 numbers below 2^128 the sum stays below 2^118, and of a sum beyond 2^128 it is above 2^-32, beside which squares that vanish count nothing.
template <typename F>
__device__ __forceinline__ float inverse_root(float sum, float eps, uint64_t cols, F squares) {
  if (!(sum <= FLT_MAX)) {
    const float less = squares(0x1p-80f);
    return less <= FLT_MAX ? 0x1p-80f / sqrtf(less / (float)cols) : __uint_as_float(0x7FC00000u);
  }
  return 1.0f / sqrtf(sum / (float)cols + eps);
}

constexpr int kLongThreads = 1024;
constexpr int threads_of(int lanes) { return lanes > kBlock ? lanes : kBlock; }

struct NormTask {
  uint64_t all, rows, cols;  // all: of all workers
  View x, r, h, y;           // r, h: may be null; y: int8 where coded
  const float* weight;
  float eps;
  float* scale;
};

// LANES take one row and hold it, HELD times 8 columns each: x and the residual are read once, and what becomes of them written once.  The memory
// bounds it: 8192 x 4096 bfloat16 with a residual, into h and codes, 235 MB, 44 us (5.3 TB/s); 1537 x 20011 float16, rows at odd places, 123 MB, 37.  One row is a
// launch and two latencies, 3.6 us.  CODED: y is codes of the rows, with a scale for each.
template <typename T, bool CODED, int LANES, int HELD, bool NARROW>
__global__ void __launch_bounds__(threads_of(LANES), sizeof(T) == 2 && LANES == kLongThreads && HELD <= 3 ? 8 : 1) rms_norm_kernel(NormTask p) {
  constexpr int kThreads = threads_of(LANES);
  __shared__ float of_sum[kThreads / kWave][2];
  __shared__ uint32_t of_max[kThreads / kWave];
  const uint32_t lane = threadIdx.x % LANES, wave = threadIdx.x / kWave;
  static_assert(LANES == kWave || LANES == kThreads, "who meets has a row, or returns, together");
  const uint64_t index = block_number() * (kThreads / LANES) + __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
  if (index >= p.all) return;
  const Joint<LANES> joint{of_sum, of_max, threadIdx.x / LANES * (LANES / kWave), wave};
  const uint32_t m = (uint32_t)index / (uint32_t)p.rows;
  const uint64_t r = index - m * p.rows;
  const T* row = static_cast<const T*>(p.x.p) + m * p.x.pitch + r * p.x.ld;
  Eight e[HELD];
  Vec8<T> x[HELD];
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    e[k] = eight_of<NARROW>((k * LANES + lane) * 8, p.cols);
    x[k] = load_eight<T, NARROW>(row, e[k], p.cols);
  }
  if (p.r.p != nullptr) {
    const T* other = static_cast<const T*>(p.r.p) + m * p.r.pitch + r * p.r.ld;
    Vec8<T> o[HELD];
#pragma unroll
    for (int k = 0; k < HELD; ++k) o[k] = load_eight<T, NARROW>(other, e[k], p.cols);
#pragma unroll
    for (int k = 0; k < HELD; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[k][i] = (T)pinned((float)x[k][i] + (float)o[k][i]);  // (h: what it is stored as is what is normalised)
  }
  // (the row is held as it was loaded, and widened where it is used: what 16-bit numbers save is a second workgroup on the CU)
  auto sum_of = [&](float f) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const float v = NARROW || i >= e[k].shift ? (float)x[k][i] * f : 0.f;
        sum += v * v;
      }
      asm volatile("" : "+v"(x[k]));
    }
    return joint.sum(sum);
  };
  const float s = inverse_root(sum_of(1.f), p.eps, p.cols, sum_of);
  if (p.h.p != nullptr) {
    T* h = static_cast<T*>(p.h.p) + m * p.h.pitch + r * p.h.ld;
#pragma unroll
    for (int k = 0; k < HELD; ++k) store_eight<T, NARROW>(h, e[k], p.cols, x[k]);
  }
  float v[CODED ? HELD : 1][8];
  uint32_t top = 0u;
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    float w[8];
    load_weight<NARROW>(p.weight, e[k], p.cols, w);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      float& y = v[CODED ? k : 0][i];
      y = (float)x[k][i] * s * w[i];
      if (CODED && (NARROW || i >= e[k].shift)) top = max(top, magnitude_bits(y));
    }
    if (!CODED) store_eight<T, NARROW>(static_cast<T*>(p.y.p) + m * p.y.pitch + r * p.y.ld, e[k], p.cols, narrowed<T>(v[0]));
  }
  if (!CODED) return;
  top = joint.max_bits(top);
  const float inv = code_inverse(top);
  if (lane == 0) p.scale[index] = code_step(top);
  int8_t* out = static_cast<int8_t*>(p.y.p) + m * p.y.pitch + r * p.y.ld;
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = code_nearest(v[CODED ? k : 0][i], inv);
    Vec8<int8_t> codes;
    const uint32_t low = pack4(q[0], q[1], q[2], q[3]), high = pack4(q[4], q[5], q[6], q[7]);
    __builtin_memcpy(&codes, &low, 4);
    __builtin_memcpy(reinterpret_cast<char*>(&codes) + 4, &high, 4);
    store_eight<int8_t, NARROW>(out, e[k], p.cols, codes);
  }
}

// Longer rows, a workgroup each: h is made (and read) again for y, and for codes once more, mostly from a cache.

template <typename T, bool CODED>
__global__ void __launch_bounds__(kLongThreads) rms_norm_long_kernel(NormTask p) {
  __shared__ float of_sum[kLongThreads / kWave][2];
  __shared__ uint32_t of_max[kLongThreads / kWave];
  const Joint<kLongThreads> joint{of_sum, of_max, 0, threadIdx.x / kWave};
  const uint64_t index = block_number();
  if (index >= p.all) return;
  const uint32_t m = (uint32_t)index / (uint32_t)p.rows;
  const uint64_t r = index - m * p.rows;
  const T* row = static_cast<const T*>(p.x.p) + m * p.x.pitch + r * p.x.ld;
  const T* other = p.r.p == nullptr ? nullptr : static_cast<const T*>(p.r.p) + m * p.r.pitch + r * p.r.ld;
  T* h = p.h.p == nullptr ? nullptr : static_cast<T*>(p.h.p) + m * p.h.pitch + r * p.h.ld;
  // A lane's own eight columns every time, so that its h may lie where x or the residual did; kept: h is there already.
  auto value = [&](uint64_t c, bool kept, Eight& e, float (&v)[8]) {
    e = eight_of<false>(c, p.cols);
    Vec8<T> x = load_eight<T, false>(kept ? h : row, e, p.cols);
    if (other != nullptr && !kept) {
      const Vec8<T> o = load_eight<T, false>(other, e, p.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (T)pinned((float)x[i] + (float)o[i]);
    }
    widen<T>(x, v);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < e.shift) v[i] = 0.f;
    return x;
  };
  Eight e;
  float v[8], sum = 0.f;
#pragma unroll 2
  for (uint64_t c = threadIdx.x * 8; c < p.cols; c += kLongThreads * 8) {
    const Vec8<T> x = value(c, false, e, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += v[i] * v[i];
    if (h != nullptr) store_eight<T, false>(h, e, p.cols, x);
  }
  sum = joint.sum(sum);
  const bool kept = h != nullptr;
  const float s = inverse_root(sum, p.eps, p.cols, [&](float f) {
    float less = 0.f;
    for (uint64_t c = threadIdx.x * 8; c < p.cols; c += kLongThreads * 8) {
      value(c, kept, e, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) less += v[i] * f * (v[i] * f);
    }
    return joint.sum(less);
  });
  auto scaled = [&](uint64_t c) {
    value(c, kept, e, v);
    float w[8];
    load_weight<false>(p.weight, e, p.cols, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] * s * w[i];
  };
  uint32_t top = 0u;
#pragma unroll 2
  for (uint64_t c = threadIdx.x * 8; c < p.cols; c += kLongThreads * 8) {
    scaled(c);
    if (CODED) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(v[i]));
    } else {
      store_eight<T, false>(static_cast<T*>(p.y.p) + m * p.y.pitch + r * p.y.ld, e, p.cols, narrowed<T>(v));
    }
  }
  if (!CODED) return;
  top = joint.max_bits(top);
  const float inv = code_inverse(top);
  if (threadIdx.x == 0) p.scale[index] = code_step(top);
#pragma unroll 2
  for (uint64_t c = threadIdx.x * 8; c < p.cols; c += kLongThreads * 8) {
    scaled(c);
    Vec8<int8_t> codes;
#pragma unroll
    for (int i = 0; i < 8; ++i) codes[i] = (int8_t)code_nearest(v[i], inv);
    store_eight<int8_t, false>(static_cast<int8_t*>(p.y.p) + m * p.y.pitch + r * p.y.ld, e, p.cols, codes);
  }
}

constexpr std::integral_constant<int, 1> kOne;
constexpr std::integral_constant<int, 2> kTwo;
constexpr std::integral_constant<int, 3> kThree;
constexpr std::integral_constant<int, 4> kFour;
constexpr std::integral_constant<int, kWave> kOfWave;
constexpr std::integral_constant<int, kBlock> kOfBlock;
constexpr std::integral_constant<int, 512> kOfSome;
constexpr std::integral_constant<int, 1024> kOfMany;

template <typename T, bool CODED>
void norm_typed(const NormTask& p, hipStream_t s) {
  auto launch = [&](auto lanes, auto held, auto narrow) {
    constexpr int threads = threads_of(lanes), each = threads / lanes;
    rms_norm_kernel<T, CODED, lanes, held, narrow><<<grid_of((p.all + each - 1) / each), threads, 0, s>>>(p);
  };
  const bool many = p.all >= 1024;  // (few rows get a workgroup each, for their latency)
  if (p.cols < 8)
    launch(kOfWave, kOne, std::true_type{});
  else if (p.cols <= 512)
    launch(kOfWave, kOne, std::false_type{});
  else if (many && p.cols <= 1024)
    launch(kOfWave, kTwo, std::false_type{});
  else if (many && p.cols <= 2048)
    launch(kOfWave, kFour, std::false_type{});
  else if (p.cols <= 2048)
    launch(kOfBlock, kOne, std::false_type{});
  else if (p.cols <= 4096)
    launch(kOfBlock, kTwo, std::false_type{});
  else if (p.cols <= 6144)
    launch(kOfBlock, kThree, std::false_type{});
  else if (p.cols <= 8192)
    launch(kOfBlock, kFour, std::false_type{});
  else if (p.cols <= 16384)
    launch(kOfMany, kTwo, std::false_type{});
  else if (p.cols <= 24576)
    launch(kOfMany, kThree, std::false_type{});
  else if (p.cols <= 32768)
    launch(kOfMany, kFour, std::false_type{});
  else
    rms_norm_long_kernel<T, CODED><<<grid_of(p.all), kLongThreads, 0, s>>>(p);
}

// ---- the gradient
//
//   s = 1 / sqrt(mean h^2 + eps),  g = w dy,  dx = s (g - h s^2 mean(g h)) + dr,  dw = sum over a worker's rows of dy h s
//
// s is made again: both sums of a row come out of the one pass that has to read it anyway.  dw lies in registers while a group of LANES takes rows, one
// after another, and the groups' parts meet in the second kernel.  4 x 2048 x 4096 bfloat16 with dr, 268 MB, 49 us (5.5 TB/s), and 5 for the parts.

struct NormGradTask {
  uint64_t rows, cols;
  View dy, h, r, dx;  // r: may be null
  const float* weight;
  float eps;
  float* part;      // [worker][parts][cols], or null: dw is not wanted
  uint32_t parts;   // workgroups of a worker
  float* row_part;  // long rows: [worker][rows][2], s and s^3 mean(g h)
};

template <typename T, int LANES, int HELD, bool NARROW>
__global__ void __launch_bounds__(threads_of(LANES)) rms_norm_grad_kernel(NormGradTask p) {
  constexpr int kThreads = threads_of(LANES), kGroups = kThreads / LANES;
  constexpr bool kAhead = LANES <= kBlock;  // the next row is on its way while one is worked on (more lanes have no registers for it)
  __shared__ float of_sum[kThreads / kWave][2];
  __shared__ float of_dw[kGroups > 1 ? kGroups - 1 : 1][kGroups > 1 ? LANES * HELD * 8 : 1];
  const uint32_t lane = threadIdx.x % LANES, group = __builtin_amdgcn_readfirstlane(threadIdx.x / LANES), wave = threadIdx.x / kWave, m = blockIdx.y;
  const Joint<LANES> joint{of_sum, nullptr, group * (LANES / kWave), wave};
  Eight e[HELD];
  float w[HELD][8], dw[HELD][8];
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    e[k] = eight_of<NARROW>((k * LANES + lane) * 8, p.cols);
    load_weight<NARROW>(p.weight, e[k], p.cols, w[k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
  }
  struct Row {
    Vec8<T> dy[HELD], h[HELD], r[HELD];
  };
  const T* dys = static_cast<const T*>(p.dy.p) + m * p.dy.pitch;
  const T* hs = static_cast<const T*>(p.h.p) + m * p.h.pitch;
  const T* rs = p.r.p == nullptr ? nullptr : static_cast<const T*>(p.r.p) + m * p.r.pitch;
  auto ask = [&](uint64_t row, Row& a) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) a.dy[k] = load_eight<T, NARROW>(dys + row * p.dy.ld, e[k], p.cols);
#pragma unroll
    for (int k = 0; k < HELD; ++k) a.h[k] = load_eight<T, NARROW>(hs + row * p.h.ld, e[k], p.cols);
    if (rs != nullptr) {
#pragma unroll
      for (int k = 0; k < HELD; ++k) a.r[k] = load_eight<T, NARROW>(rs + row * p.r.ld, e[k], p.cols);
    }
  };
  // A workgroup's rows lie kGroups parts apart; the groups of one make as many turns, those past the end without a row (the last row again,
  // which is not counted).
  const uint64_t step = (uint64_t)p.parts * kGroups;
  uint64_t row = (uint64_t)blockIdx.x * kGroups + group;
  Row now, next;
  if (kAhead) ask(min(row, p.rows - 1), now);
  for (uint64_t first = (uint64_t)blockIdx.x * kGroups; first < p.rows; first += step, row += step) {
    const bool in = row < p.rows;
    if (kAhead)
      ask(min(row + step, p.rows - 1), next);  // (of a row that another workgroup may be writing, where results lie on inputs: then it is not used)
    else
      ask(min(row, p.rows - 1), now);
    auto keep = [&]() {
#pragma unroll
      for (int k = 0; k < HELD; ++k) {
        asm volatile("" : "+v"(now.dy[k]));
        asm volatile("" : "+v"(now.h[k]));
      }
    };
    float squares = 0.f, dot = 0.f;
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const bool mine = NARROW || i >= e[k].shift;
        const float h = mine ? (float)now.h[k][i] : 0.f, dy = mine ? (float)now.dy[k][i] : 0.f;
        squares += h * h;
        dot += dy * w[k][i] * h;
      }
    }
    keep();
    joint.sum(squares, dot);
    float over = 1.f;  // (what the dot product is taken down by where squares leave binary32)
    const float s = inverse_root(squares, p.eps, p.cols, [&](float f) {
      float less = 0.f, small = 0.f;
#pragma unroll
      for (int k = 0; k < HELD; ++k) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          const bool mine = NARROW || i >= e[k].shift;
          const float h = mine ? (float)now.h[k][i] * f : 0.f;
          less += h * h;
          small += (mine ? (float)now.dy[k][i] : 0.f) * w[k][i] * h;
        }
      }
      joint.sum(less, small);
      dot = small;
      over = f;
      return less;
    });
    // (here the operands are what was loaded, and no longer also what the sums made of them: that would not fit the registers)
    keep();
    // mean(g h s), the part of g along h
    const float along = dot * (s / over) / (float)p.cols;
    if (in) {
      T* dx = static_cast<T*>(p.dx.p) + m * p.dx.pitch + row * p.dx.ld;
#pragma unroll
      for (int k = 0; k < HELD; ++k) {
        float v[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          const float unit = (float)now.h[k][i] * s, dy = (float)now.dy[k][i];
          dw[k][i] += dy * unit;
          v[i] = s * (dy * w[k][i] - unit * along);
          if (rs != nullptr) v[i] += (float)now.r[k][i];
        }
        store_eight<T, NARROW>(dx, e[k], p.cols, narrowed<T>(v));
        if (!kAhead) __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (kAhead) now = next;
  }
  if (p.part == nullptr) return;
  if (kGroups > 1) {
    if (group > 0) {
#pragma unroll
      for (int k = 0; k < HELD; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) of_dw[group - 1][(k * 8 + i) * LANES + lane] = dw[k][i];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < HELD; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int g = 0; g + 1 < kGroups; ++g) dw[k][i] += of_dw[g][(k * 8 + i) * LANES + lane];
  }
  float* to = p.part + ((uint64_t)m * p.parts + blockIdx.x) * p.cols;
#pragma unroll
  for (int k = 0; k < HELD; ++k) {
    Vec8<float> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = dw[k][i];
    store_eight<float, NARROW>(to, e[k], p.cols, v);
  }
}

// Longer rows: a row's two sums by a workgroup, then columns, by tiles of a workgroup's eights (1537 x 20011 float16: 30 and 32 us).
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rms_norm_grad_sums_kernel(NormGradTask p, uint64_t rows) {
  __shared__ float of_sum[kLongThreads / kWave][2];
  const Joint<kLongThreads> joint{of_sum, nullptr, 0, threadIdx.x / kWave};
  const uint64_t index = block_number();
  if (index >= rows) return;
  const uint32_t m = (uint32_t)index / (uint32_t)p.rows;
  const uint64_t r = index - m * p.rows;
  const T* dys = static_cast<const T*>(p.dy.p) + m * p.dy.pitch + r * p.dy.ld;
  const T* hs = static_cast<const T*>(p.h.p) + m * p.h.pitch + r * p.h.ld;
  float dot;
  auto sums = [&](float f) {
    float squares = 0.f;
    dot = 0.f;
#pragma unroll 2
    for (uint64_t c = threadIdx.x * 8; c < p.cols; c += kLongThreads * 8) {
      const Eight e = eight_of<false>(c, p.cols);
      float dy[8], h[8], w[8];
      widen<T>(load_eight<T, false>(dys, e, p.cols), dy);
      widen<T>(load_eight<T, false>(hs, e, p.cols), h);
      load_weight<false>(p.weight, e, p.cols, w);
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const float v = i >= e.shift ? h[i] * f : 0.f;
        squares += v * v;
        dot += (i >= e.shift ? dy[i] : 0.f) * w[i] * v;
      }
    }
    joint.sum(squares, dot);
    return squares;
  };
  float over = 1.f;
  const float all = sums(1.f);
  const float s = inverse_root(all, p.eps, p.cols, [&](float f) {
    over = f;
    return sums(f);
  });
  if (threadIdx.x == 0) {
    p.row_part[2 * index] = s;
    p.row_part[2 * index + 1] = dot * (s / over) / (float)p.cols;
  }
}

template <typename T>
__global__ void __launch_bounds__(kBlock) rms_norm_grad_columns_kernel(NormGradTask p) {
  const uint32_t m = blockIdx.z;
  const uint64_t c = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) * 8;
  if (c >= p.cols) return;
  const Eight e = eight_of<false>(c, p.cols);
  float w[8], dw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  load_weight<false>(p.weight, e, p.cols, w);
#pragma unroll 2
  for (uint64_t r = blockIdx.y; r < p.rows; r += p.parts) {
    const float s = p.row_part[2 * (m * p.rows + r)], along = p.row_part[2 * (m * p.rows + r) + 1];
    float dy[8], h[8], v[8];
    widen<T>(load_eight<T, false>(static_cast<const T*>(p.dy.p) + m * p.dy.pitch + r * p.dy.ld, e, p.cols), dy);
    widen<T>(load_eight<T, false>(static_cast<const T*>(p.h.p) + m * p.h.pitch + r * p.h.ld, e, p.cols), h);
    if (p.r.p != nullptr)
      widen<T>(load_eight<T, false>(static_cast<const T*>(p.r.p) + m * p.r.pitch + r * p.r.ld, e, p.cols), v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float unit = h[i] * s, x = s * (dy[i] * w[i] - unit * along);
      dw[i] += dy[i] * unit;
      v[i] = p.r.p != nullptr ? x + v[i] : x;
    }
    store_eight<T, false>(static_cast<T*>(p.dx.p) + m * p.dx.pitch + r * p.dx.ld, e, p.cols, narrowed<T>(v));
  }
  if (p.part == nullptr) return;
  Vec8<float> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = dw[i];
  store_eight<float, false>(p.part + ((uint64_t)m * p.parts + blockIdx.y) * p.cols, e, p.cols, v);
}

// dw of a worker: its parts in order, a quarter of them by each wavefront.
__global__ void __launch_bounds__(kBlock) rms_norm_grad_join_kernel(const float* part, uint32_t parts, uint64_t cols, float* dw) {
  constexpr uint32_t kWaves = kBlock / kWave;
  __shared__ float of_wave[kWaves][kWave];
  const uint32_t m = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint64_t c = (uint64_t)blockIdx.x * kWave + lane, at = min(c, cols - 1);
  const uint32_t each = (parts + kWaves - 1) / kWaves, first = wave * each, end = min(parts, first + each);
  float sum = 0.f;
#pragma unroll 8
  for (uint32_t k = first; k < end; ++k) sum += part[((uint64_t)m * parts + k) * cols + at];
  of_wave[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || c >= cols) return;
  for (uint32_t k = 1; k < kWaves; ++k) sum += of_wave[k][lane];
  dw[m * cols + c] = sum;
}

// How long a row the workgroups hold: for longer ones they would have no registers but for one on a CU.  (1537 x 20011 bfloat16, 184 MB, 73 us, where two passes
// take 71; 8 x 100 x 18000 40 and 32; 2048 x 16384 52 and 64.)
constexpr uint64_t kHeldCols = 16384;

// So many rows one after another take less than parts that have to be joined, by a launch more: 8 rows of 1000 bfloat16, two for each wavefront, 4.8 us and 5.6, 2
// of 4096 4.7 and 5.4 (four after another 7.6 and 5.4).
constexpr uint64_t kTurns = 2;

// Workgroups of a worker: as many as run at a time, but no more than there are rows for.
uint32_t grad_parts(const Extent& n) {
  const uint64_t groups = n.cols <= 1024 ? kBlock / kWave : 1;  // rows that a workgroup has at a time
  // (268 MB of bfloat16, us, with 256 / 512 / 768 / 1024 workgroups: 65536 x 256 (half of that) 79 / 53 / 48 / 48, 8192 x 4096 75 / 54 / 53 / 55, 4096 x 8192
  // 59 / 56 / 69 / 68, 2048 x 16384 64 / 71 / 81 / 87)
  const uint64_t most = n.cols <= 512 ? 1024 : n.cols <= 1024 ? 512 : n.cols <= 4096 ? 768 : n.cols <= 8192 ? 512 : n.cols <= kHeldCols ? 256 : 512;
  const uint64_t tiles = n.cols > kHeldCols ? (n.cols + kBlock * 8 - 1) / (kBlock * 8) : 1;
  const uint64_t each = std::max<uint64_t>(1, most / (n.workers * tiles)), rows = (n.rows + groups - 1) / groups;
  if (rows <= kTurns) return 1;
  return (uint32_t)std::min(each, rows);
}

template <typename T>
void norm_grad_typed(uint32_t workers, const NormGradTask& p, hipStream_t s) {
  auto launch = [&](auto lanes, auto held, auto narrow) {
    rms_norm_grad_kernel<T, lanes, held, narrow><<<dim3(p.parts, workers), threads_of(lanes), 0, s>>>(p);
  };
  if (p.cols > kHeldCols) {
    rms_norm_grad_sums_kernel<T><<<grid_of(workers * p.rows), kLongThreads, 0, s>>>(p, workers * p.rows);
    rms_norm_grad_columns_kernel<T><<<dim3((uint32_t)((p.cols + kBlock * 8 - 1) / (kBlock * 8)), p.parts, workers), kBlock, 0, s>>>(p);
  } else if (p.cols < 8) {
    launch(kOfWave, kOne, std::true_type{});
  } else if (p.cols <= 512) {
    launch(kOfWave, kOne, std::false_type{});
  } else if (p.cols <= 1024) {
    launch(kOfWave, kTwo, std::false_type{});
  } else if (p.cols <= 2048) {
    launch(kOfBlock, kOne, std::false_type{});
  } else if (p.cols <= 4096) {
    launch(kOfBlock, kTwo, std::false_type{});
  } else if (p.cols <= 6144) {
    launch(kOfBlock, kThree, std::false_type{});
  } else if (p.cols <= 8192) {
    launch(kOfBlock, kFour, std::false_type{});
  } else {
    launch(kOfSome, kFour, std::false_type{});
  }
}

}  // namespace

hipError_t launch_rms_norm(tng_type type, const Extent& n, const View& x, const View& residual, const NormArgs& norm, const View& h, const View& y,
                           float* scale, hipStream_t s) {
  const NormTask p{n.workers * n.rows, n.rows, n.cols, x, residual, h, y, norm.weight, norm.eps, scale};
  const bool coded = scale != nullptr;
  switch (type) {
    case TNG_TYPE_F32: coded ? norm_typed<float, true>(p, s) : norm_typed<float, false>(p, s); break;
    case TNG_TYPE_BF16: coded ? norm_typed<bf16_t, true>(p, s) : norm_typed<bf16_t, false>(p, s); break;
    default: coded ? norm_typed<f16_t, true>(p, s) : norm_typed<f16_t, false>(p, s); break;
  }
  return hipGetLastError();
}

size_t rms_norm_grad_floats(const Extent& n) {
  return n.workers * ((uint64_t)grad_parts(n) * n.cols + (n.cols > kHeldCols ? 2 * n.rows : 0));
}

hipError_t launch_rms_norm_grad(tng_type type, const Extent& n, const View& dy, const View& h, const View& residual, const NormArgs& norm,
                                const View& dx, float* dw, float* scratch, hipStream_t s) {
  const uint32_t parts = grad_parts(n);
  NormGradTask p{n.rows, n.cols, dy, h, residual, dx, norm.weight, norm.eps, dw == nullptr ? nullptr : scratch, parts, nullptr};
  p.row_part = scratch + (uint64_t)n.workers * parts * n.cols;
  const bool joined = dw != nullptr && (parts > 1 || n.rows == 0);  // (one part is dw itself)
  if (!joined) p.part = dw;
  if (n.rows > 0) {
    switch (type) {
      case TNG_TYPE_F32: norm_grad_typed<float>(n.workers, p, s); break;
      case TNG_TYPE_BF16: norm_grad_typed<bf16_t>(n.workers, p, s); break;
      default: norm_grad_typed<f16_t>(n.workers, p, s); break;
    }
  }
  if (joined)
    rms_norm_grad_join_kernel<<<dim3((uint32_t)((n.cols + kWave - 1) / kWave), n.workers), kBlock, 0, s>>>(scratch, n.rows > 0 ? parts : 0u, n.cols,
                                                                                                     dw);
  return hipGetLastError();
}

}  // namespace tng
