// Products of 8-bit codes on the matrix units (gfx950): y = a_scale b_scale (a b^T) + bias, sums in 32-bit integers.
#include "tng_layer_device.hpp"

namespace tng {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// Sums of 2^16 products of two codes (127^2 each, or 128^2) stay inside 32 bits; a deeper product is split, and its pieces are joined in
// 64 bits.
constexpr uint64_t kMaxDepth = 1ull << 16;

// What a workgroup knows of the product.
struct Task {
  uint32_t rows_of_worker;         // of a, for dropout's draws; the product's own rows may be those of all workers together
  uint64_t rows, channels, depth;  // of this launch's matrices
  View a, b, y, x;
  const float *a_scale, *b_scale, *bias;
  uint64_t b_scale_pitch;
  uint64_t split_depth;  // depth of a split
  uint32_t splits;
  int32_t* parts;  // [split][worker][rows][channels], or null: the kernel finishes y itself
  DropArgs drop;
  int drops;  // the tail is wanted
};

// y of one element from its sum, before the rounding to y's type.
__device__ __forceinline__ float scaled(float sum, float a_scale, float b_scale, float bias) { return sum * a_scale * b_scale + bias; }

// keep f'(x) / (1 - p) of element (t, n).
template <typename T>
__device__ __forceinline__ float tail(float y, const Task& p, uint32_t m, uint64_t t, uint64_t n) {
  if (!p.drops) return y;
  const uint32_t w = p.rows == p.rows_of_worker ? m : (uint32_t)(t / p.rows_of_worker);
  const uint64_t e = (t - (uint64_t)(w - m) * p.rows_of_worker) * p.channels + n;
  uint32_t word = 0u;
  if (p.drop.threshold != 0u) {
    const U32x4 v = philox4x32_10((uint32_t)(e >> 2), w, p.drop.iter, p.drop.word, p.drop.k0, p.drop.k1);
    const uint32_t k = (uint32_t)e & 3u;
    word = k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w;
  }
  bool pass = kept(word, p.drop);
  if (p.drop.relu) pass = pass && !((float)static_cast<const T*>(p.x.p)[m * p.x.pitch + t * p.x.ld + n] <= 0.f);
  return pass ? y * p.drop.scale : 0.f;
}

template <typename T>
__device__ __forceinline__ void finish(float sum, const Task& p, uint32_t m, uint64_t t, uint64_t n) {
  const float sa = p.a_scale != nullptr ? p.a_scale[m * p.rows + t] : 1.f;
  const float sb = p.b_scale != nullptr ? p.b_scale[m * p.b_scale_pitch + n] : 1.f;
  const float bias = p.bias != nullptr ? p.bias[n] : 0.f;
  const float y = tail<T>(scaled(sum, sa, sb, bias), p, m, t, n);
  static_cast<T*>(p.y.p)[m * p.y.pitch + t * p.y.ld + n] = (T)y;
}

// Any alignment, any size: 64 x 64 results for a workgroup, 32 x 32 for each of its wavefronts, 64 codes deep at a time through LDS.
constexpr int kAnyTile = 64, kAnyDepth = 64;

// Codes k .. k + 15 of a row, 0 past `end`.
__device__ __forceinline__ v4i load16_any(const int8_t* row, uint64_t k, uint64_t end) {
  typedef int four __attribute__((ext_vector_type(4), aligned(1)));
  v4i v = {0, 0, 0, 0};
  if (k + 16 <= end) {
    const four u = *reinterpret_cast<const four*>(row + k);
    v = u;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i)
      if (k + i < end) v[i / 4] |= (int)((uint32_t)(uint8_t)row[k + i] << (i % 4 * 8));
  }
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kBlock) product_any_kernel(Task p) {
  constexpr int kPitch = kAnyDepth + 16;  // bytes; the 16 keep the rows of a fragment in different banks
  __shared__ __align__(16) int8_t tile_a[kAnyTile * kPitch];
  __shared__ __align__(16) int8_t tile_b[kAnyTile * kPitch];
  const uint32_t m = blockIdx.y, split = blockIdx.z, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint32_t across = (uint32_t)((p.channels + kAnyTile - 1) / kAnyTile);
  const uint64_t t0 = (uint64_t)(blockIdx.x / across) * kAnyTile, n0 = (uint64_t)(blockIdx.x % across) * kAnyTile;
  const uint64_t begin = split * p.split_depth, end = min(p.depth, begin + p.split_depth);
  const uint32_t row = threadIdx.x / 4, piece = threadIdx.x % 4;
  const int8_t* a = static_cast<const int8_t*>(p.a.p) + m * p.a.pitch + min(t0 + row, p.rows - 1) * p.a.ld;
  const int8_t* b = static_cast<const int8_t*>(p.b.p) + m * p.b.pitch + min(n0 + row, p.channels - 1) * p.b.ld;
  v4i sum[2][2] = {};
  for (uint64_t k = begin; k < end; k += kAnyDepth) {
    const v4i va = load16_any(a, k + piece * 16, end), vb = load16_any(b, k + piece * 16, end);
    __syncthreads();
    *reinterpret_cast<v4i*>(tile_a + row * kPitch + piece * 16) = va;
    *reinterpret_cast<v4i*>(tile_b + row * kPitch + piece * 16) = vb;
    __syncthreads();
    // the channels are the rows of the unit's result: a lane holds four of them, one after another, of one token
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const v4i fb = *reinterpret_cast<const v4i*>(tile_b + ((wave % 2) * 32 + i * 16 + lane % 16) * kPitch + lane / 16 * 16);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const v4i fa = *reinterpret_cast<const v4i*>(tile_a + ((wave / 2) * 32 + j * 16 + lane % 16) * kPitch + lane / 16 * 16);
        sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb, fa, sum[i][j], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint64_t t = t0 + (wave / 2) * 32 + j * 16 + lane % 16, n = n0 + (wave % 2) * 32 + i * 16 + lane / 16 * 4 + r;
        if (t >= p.rows || n >= p.channels) continue;
        if (p.parts != nullptr)
          p.parts[(((uint64_t)split * gridDim.y + m) * p.rows + t) * p.channels + n] = sum[i][j][r];
        else
          finish<T>((float)sum[i][j][r], p, m, t, n);
      }
}

// The splits' sums joined.
template <typename T>
__global__ void __launch_bounds__(kBlock) product_join_kernel(Task p, uint32_t workers) {
  const uint64_t n = p.rows * p.channels, e = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
  const uint32_t m = blockIdx.y;
  if (e >= n) return;
  int64_t sum = 0;
  for (uint32_t s = 0; s < p.splits; ++s) sum += p.parts[((uint64_t)s * workers + m) * n + e];
  finish<T>((float)sum, p, m, e / p.channels, e % p.channels);
}

struct Plan {
  uint32_t splits;
  uint64_t split_depth;
};

Plan plan_of(const Product& p) {
  Plan plan;
  plan.splits = (uint32_t)((p.depth + kMaxDepth - 1) / kMaxDepth);
  if (plan.splits == 0) plan.splits = 1;
  plan.split_depth = plan.splits == 1 ? p.depth : kMaxDepth;
  return plan;
}

template <typename T>
hipError_t product_typed(const Product& p, void* scratch, hipStream_t s) {
  const Plan plan = plan_of(p);
  Task t{};
  t.rows_of_worker = (uint32_t)p.rows;
  t.rows = p.rows;
  t.channels = p.channels;
  t.depth = p.depth;
  t.a = p.a;
  t.b = p.b;
  t.y = p.y;
  t.x = p.x;
  t.a_scale = p.a_scale;
  t.b_scale = p.b_scale;
  t.bias = p.bias;
  t.b_scale_pitch = p.b_scale_pitch;
  t.split_depth = plan.split_depth;
  t.splits = plan.splits;
  t.parts = plan.splits > 1 ? static_cast<int32_t*>(scratch) : nullptr;
  if (p.drop != nullptr) {
    t.drop = *p.drop;
    t.drops = 1;
  }
  const uint64_t tiles = ((p.rows + kAnyTile - 1) / kAnyTile) * ((p.channels + kAnyTile - 1) / kAnyTile);
  product_any_kernel<T><<<dim3((uint32_t)tiles, p.workers, plan.splits), kBlock, 0, s>>>(t);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || plan.splits == 1) return e;
  const dim3 grid((uint32_t)((p.rows * p.channels + kBlock - 1) / kBlock), p.workers);
  product_join_kernel<T><<<grid, kBlock, 0, s>>>(t, p.workers);
  return hipGetLastError();
}

}  // namespace

size_t product_scratch_bytes(const Product& p) {
  const Plan plan = plan_of(p);
  return plan.splits > 1 ? plan.splits * (size_t)p.workers * p.rows * p.channels * sizeof(int32_t) : 0;
}

hipError_t launch_product(const Product& p, void* scratch, hipStream_t s) {
  switch (p.type) {
    case TNG_TYPE_F32: return product_typed<float>(p, scratch, s);
    case TNG_TYPE_BF16: return product_typed<bf16_t>(p, scratch, s);
    default: return product_typed<f16_t>(p, scratch, s);
  }
}

}  // namespace tng
