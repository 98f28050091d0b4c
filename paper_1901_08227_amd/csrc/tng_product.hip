// Products of 8-bit codes on the matrix units (gfx950): y = a_scale b_scale (a b^T) + bias, sums in 32-bit integers.
#include "tng_layer_device.hpp"

#include <algorithm>
#include <type_traits>

namespace tng {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// Sums of 2^16 products of two codes (127^2 each, or 128^2) stay inside 32 bits; a deeper product is split, and its pieces are joined in
// 64 bits.
constexpr uint64_t kMaxDepth = 1ull << 16;

// What a workgroup knows of the product.
struct Task {
  uint32_t workers;
  uint32_t rows_of_worker;         // of a, for dropout's draws; the product's own rows may be those of all workers together
  uint64_t rows, channels, depth;  // of this launch's matrices
  View a, b, y, x;
  const float *a_scale, *b_scale, *bias;
  uint64_t b_scale_pitch;
  uint64_t split_depth;  // depth of a split
  uint32_t splits;
  int32_t* parts;  // [split][worker][rows][part_pitch], or null: the kernel finishes y itself
  uint32_t part_pitch;
  DropArgs drop;
  int drops;  // the tail is wanted
};

// y of one element from its sum, before the rounding to y's type.
__device__ __forceinline__ float scaled(float sum, float a_scale, float b_scale, float bias) { return sum * a_scale * b_scale + bias; }

// The worker that row t of the product belongs to, and its row there.
__device__ __forceinline__ uint32_t worker_of(const Task& p, uint32_t m, uint32_t* t) {
  if (p.rows == p.rows_of_worker) return m;
  const uint32_t w = *t / p.rows_of_worker;  // (m is 0: the rows of all workers)
  *t -= w * p.rows_of_worker;
  return w;
}

// keep f'(x) / (1 - p) of element (t, n).
template <typename T>
__device__ __forceinline__ float tail(float y, const Task& p, uint32_t m, uint64_t t, uint64_t n) {
  if (!p.drops) return y;
  uint32_t row = (uint32_t)t;
  const uint32_t w = worker_of(p, m, &row);
  const uint64_t e = (uint64_t)row * p.channels + n;
  uint32_t word = 0u;
  if (p.drop.threshold != 0u) {
    const U32x4 v = philox4x32_10((uint32_t)(e >> 2), w, p.drop.iter, p.drop.word, p.drop.k0, p.drop.k1);
    const uint32_t k = (uint32_t)e & 3u;
    word = k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w;
  }
  bool pass = kept(word, p.drop);
  if (p.drop.relu) pass = pass && !((float)static_cast<const T*>(p.x.p)[w * p.x.pitch + (uint64_t)row * p.x.ld + n] <= 0.f);
  return pass ? y * p.drop.scale : 0.f;
}

// The same of N consecutive channels from n on; x: what relu was taken of, t: the row among worker w's.
template <int N>
__device__ __forceinline__ void tail_n(float (&y)[N], const float (&x)[N], const Task& p, uint32_t w, uint64_t t, uint64_t n) {
  const uint64_t e = t * p.channels + n;
#pragma unroll
  for (int b = 0; b < N; b += 4) {  // (a block at a time: the sums leave few registers)
    uint32_t word[4] = {0u, 0u, 0u, 0u};
    if (p.drop.threshold != 0u) draw_n<4>(e + b, (p.channels & 3u) == 0u, w, p.drop, word);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[b + i] = kept(word[i], p.drop) && !(x[b + i] <= 0.f) ? y[b + i] * p.drop.scale : 0.f;
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <typename T, int N>
__device__ __forceinline__ void load_gate(float (&x)[N], const Task& p, uint32_t w, uint64_t t, uint64_t n, uint64_t left) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = 1.f;
  if (p.drop.relu) load_n_within<T, N>(static_cast<const T*>(p.x.p) + w * p.x.pitch + t * p.x.ld + n, left, 1.f, x);
}

template <typename T>
__device__ __forceinline__ void finish(float sum, const Task& p, uint32_t m, uint64_t t, uint64_t n) {
  const float sa = p.a_scale != nullptr ? p.a_scale[m * p.rows + t] : 1.f;
  const float sb = p.b_scale != nullptr ? p.b_scale[m * p.b_scale_pitch + n] : 1.f;
  const float bias = p.bias != nullptr ? p.bias[n] : 0.f;
  const float y = tail<T>(scaled(sum, sa, sb, bias), p, m, t, n);
  static_cast<T*>(p.y.p)[m * p.y.pitch + t * p.y.ld + n] = (T)y;
}

// Workgroups go to the eight dies in turn, and each die has its own cache: it takes a run of tiles that lie together, and its workgroups
// take those in turn.
struct Run {
  uint32_t first, end, step;
};
__device__ __forceinline__ Run run_of(uint32_t block, uint32_t blocks, uint32_t tiles) {
  constexpr uint32_t kDies = 8;
  const uint32_t die = block % kDies, each = tiles / kDies, more = tiles % kDies, begin = die * each + min(die, more);
  return Run{begin + block / kDies, begin + each + (die < more ? 1u : 0u), (blocks - die + kDies - 1) / kDies};
}

// In a matrix, tiles follow each other down columns of kGroup tiles of tokens: what is worked on at a time is about square.
__device__ __forceinline__ void place_in_plane(uint32_t tile, uint32_t across, uint32_t down, uint32_t* n, uint32_t* t) {
  constexpr uint32_t kGroup = 4;
  const uint32_t group = tile / (kGroup * across), first = group * kGroup, high = min(kGroup, down - first);
  const uint32_t in = tile - group * kGroup * across;
  *t = first + in % high;
  *n = in / high;
}

// Any alignment, any size: 64 x 64 results for a workgroup, 32 x 32 for each of its wavefronts, 64 codes deep at a time through LDS, and through
// registers on the way there (loads that go to LDS directly want aligned rows).  That way bounds it: 2048 x 2048 x 2047 45 us (0.38 POP/s; 14
// where rows are 2048 apart), 200 x 8192 x 5000 from an odd address 55 (the next 64 codes under way meanwhile; 63 without).
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
  v4i va = load16_any(a, begin + piece * 16, end), vb = load16_any(b, begin + piece * 16, end);
  for (uint64_t k = begin; k < end; k += kAnyDepth) {
    __syncthreads();
    *reinterpret_cast<v4i*>(tile_a + row * kPitch + piece * 16) = va;
    *reinterpret_cast<v4i*>(tile_b + row * kPitch + piece * 16) = vb;
    __syncthreads();
    va = load16_any(a, k + kAnyDepth + piece * 16, end);  // (the next 64, under way while these are multiplied)
    vb = load16_any(b, k + kAnyDepth + piece * 16, end);
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
          p.parts[(((uint64_t)split * gridDim.y + m) * p.rows + t) * p.part_pitch + n] = sum[i][j][r];
        else
          finish<T>((float)sum[i][j][r], p, m, t, n);
      }
}

// ---- The tile kernel: rows of a and b that begin 16-byte aligned.
//
// A workgroup makes kChannels x kTokens results at a time, 128 codes deep (a stage).  SLOTS stages of both tiles lie in LDS, filled by
// loads that go there directly.  A stage is two halves of CN groups of matrix instructions; meanwhile a wavefront reads the codes
// of the groups that follow into registers, and a stage to come is asked for, a load after each group:
//
//   first kMeet groups of stage k    | read what is left of stage k
//   wait for stage k + 1 (not for those after it); barrier: it is there for all, and stage k is in registers everywhere
//   last groups of stage k           | read the beginning of stage k + 1; ask for stage k + SLOTS, in the place of stage k
//
// A workgroup takes tiles until there are no more, and asks for the next tile's first stages before it scales and writes a tile.
//
// What bounds it: of large tiles (256 x 256: 128 operations for each byte that comes from a cache) the matrix units, at the clock that
// their power leaves.  8192 x 8192 x 8192 takes 406 us, 2.7 POP/s; the same instructions on registers alone reach 4.1 on random codes and 4.8 on
// zeros.  Of small ones and of few the time of a stage, its requests to the die's cache: 2048 x 2048 x 2048 13 us, at 300 to 370 cycles a
// request.  Rows that begin on no line of 128 bytes take up to twice as many: 200 x 8192 x 5000 23.7 us with rows 5008 apart, 18.4 with 5120.
// Stages of 128 codes are whole lines of memory where rows are (rings of 64-code stages: 8192^3 in 550 us), eight wavefronts leave each 128 x 64
// results (four of 128 x 128: 516), a load after each group keeps the memory and the matrix units busy together (two at a time: 501).
constexpr int kDepth = 128;  // bytes of a stage's rows: eight 16-byte pieces

// A tile's row has its eight 16-byte pieces moved, piece c to c ^ moved_by, so that the 16 lanes that read one piece of 16 rows meet in
// no bank (rows are 32 banks long, of 64).  Those are rows 16 a + i, or with kWide 32 (a / 2) + 8 (i / 4) + 4 (a % 2) + i % 4.
template <bool kWide>
__device__ __forceinline__ uint32_t moved_by(uint32_t row) {
  return kWide ? ((row >> 1) & 1u) | ((row >> 2) & 6u) : (row >> 1) & 7u;
}

// Of 16 codes, those whose number, k and on, is less than `end`; the others 0.
__device__ __forceinline__ v4i before(v4i v, int k, int end) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = min(max(end - (k + 4 * w), 0), 4);
    v[w] &= n == 4 ? -1 : (int)((1u << (8 * n)) - 1u);
  }
  return v;
}

// CN, TN: 16-row tiles of channels and tokens for each wavefront; CW, TW: wavefronts along each.
template <typename T, int CN, int TN, int CW, int TW, int SLOTS>
struct TileKernel {
  static constexpr int kChannels = CN * CW * 16, kTokens = TN * TW * 16, kWaves = CW * TW;
  static constexpr int kThreads = kWaves * kWave, kRows = kChannels + kTokens;
  static constexpr int kStageBytes = kRows * kDepth;
  static constexpr int kRing = SLOTS * kStageBytes;
  // behind the stages: scales and bias of the channels, scales of the tokens, of this tile and the next
  static constexpr int kFactorBytes = (2 * kChannels + kTokens) * 4, kLdsBytes = kRing + 2 * kFactorBytes;
  static constexpr int kLoads = kRows / 8 / kWaves;  // of 8 rows, for each wavefront and stage
  static constexpr int kLoadsOfB = kChannels / 8 / kWaves;
  static_assert(kChannels % (8 * kWaves) == 0 && kTokens % (8 * kWaves) == 0, "loads divide evenly");
  static constexpr int kGroups = 2 * CN, kAhead = CN > 4 ? CN - 3 : CN - 1, kMeet = kGroups - kAhead;
  static constexpr int kAsks = (kLoads + kGroups - 1) / kGroups;  // loads after each group
  static constexpr int kOther = CN > 4 ? 2 : 0;  // the group from which on the second half's tokens are read
  static_assert(kOther + TN <= kMeet && kAhead < CN, "what is read ahead has a place");
  // A lane has four channels of a tile for one token; with 16-bit results the rows are ordered so that two tiles make eight in a row.
  static constexpr bool kWide = sizeof(T) == 2;
  static constexpr int kRun = kWide ? 8 : 4, kTilesOfRun = kRun / 4;
  static_assert(CN % kTilesOfRun == 0, "tiles of channels go in pairs");
  static constexpr int kWorkgroups = 256 * (kLdsBytes <= 80 * 1024 ? 2 : 1);  // that run at a time

  static __device__ __forceinline__ uint32_t channel_row(uint32_t a, uint32_t i) {
    return kWide ? (a / 2) * 32 + i / 4 * 8 + (a % 2) * 4 + i % 4 : a * 16 + i;
  }
};

// Where a tile lies; the same for all lanes.
struct Spot {
  uint32_t m, split, channels, tokens, depth;  // channels, tokens: how many of the tile's there are
  uint64_t n0, t0;
};

template <typename K>
__device__ __forceinline__ Spot spot_of(const Task& p, uint32_t tile, uint32_t across, uint32_t down) {
  const uint32_t each = across * down, plane = tile / each, workers = p.workers;
  uint32_t tn, tt;
  place_in_plane(tile - plane * each, across, down, &tn, &tt);
  Spot s;
  s.split = plane / workers;
  s.m = plane - s.split * workers;
  s.n0 = (uint64_t)tn * K::kChannels;
  s.t0 = (uint64_t)tt * K::kTokens;
  s.channels = (uint32_t)min(p.channels - s.n0, (uint64_t)K::kChannels);
  s.tokens = (uint32_t)min(p.rows - s.t0, (uint64_t)K::kTokens);
  s.depth = (uint32_t)min(p.depth - s.split * p.split_depth, p.split_depth);
  return s;
}

// f(0), f(kStep), ... below N, each with its number known to the compiler: where a loop would be too much to unroll.
template <int N, int kStep, int kAt = 0, typename F>
__device__ __forceinline__ void each_of(F f) {
  if constexpr (kAt < N) {
    f(std::integral_constant<int, kAt>{});
    each_of<N, kStep, kAt + kStep>(f);
  }
}

// What becomes of the sums.
constexpr int kScaled = 0, kTail = 1, kParts = 2;

// Scales, bias, the tail of a gradient, and the rounding to y's type, of a wavefront's results; or their sums as they are.  factors: in LDS.
template <typename K, typename T, int END, int CN, int TN>
__device__ __forceinline__ void write_tile(const Task& p, const Spot& s, const v4i (&sum)[CN][TN], uint32_t cw, uint32_t tw, uint32_t lane,
                                           const float* factors) {
  constexpr int kRun = K::kRun;
  const uint32_t n_in = cw * CN * 16 + K::channel_row(0, lane / 16 * 4), t_in = tw * TN * 16 + lane % 16;
  const bool full = s.channels == K::kChannels && s.tokens == K::kTokens;
  // With a tail: each row's worker and its number there, and what relu was taken of, a run of channels ahead of its use.
  typedef T run_t __attribute__((ext_vector_type(kRun), aligned(alignof(T))));
  uint32_t w[TN], row[TN];
  run_t ahead[TN];
  constexpr bool kClamped = CN <= 4;  // (large tiles have no registers for it, and few of them are not whole)
  auto fetch = [&](int b, uint32_t n) {
    const T* from = static_cast<const T*>(p.x.p) + w[b] * p.x.pitch + row[b] * p.x.ld + s.n0;
    if (full) {
      ahead[b] = *reinterpret_cast<const run_t*>(from + n);
    } else if (kClamped) {  // (past the end: the last channel, for a result that goes nowhere)
#pragma unroll
      for (int r = 0; r < kRun; ++r) ahead[b][r] = from[min(n + r, s.channels - 1)];
    }
  };
  if (END == kTail) {
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      row[b] = (uint32_t)s.t0 + min(t_in + b * 16, s.tokens - 1);
      w[b] = worker_of(p, s.m, &row[b]);
      if (p.drop.relu) fetch(b, n_in);
    }
  }
  float sa[TN];
#pragma unroll
  for (int b = 0; b < TN; ++b) sa[b] = p.a_scale != nullptr ? factors[2 * K::kChannels + t_in + b * 16] : 1.f;
  each_of<CN, K::kTilesOfRun>([&](auto at) {
    constexpr int a = at;
    const uint32_t n = n_in + K::channel_row(a, 0);
    const uint64_t left = full ? kRun : n < s.channels ? s.channels - n : 0;
    if (left == 0) return;
    if (END == kParts) {
#pragma unroll
      for (int b = 0; b < TN; ++b) {
        const uint32_t t = t_in + b * 16;
        if (!full && t >= s.tokens) continue;
        int32_t* out = p.parts + (((uint64_t)s.split * p.workers + s.m) * p.rows + s.t0 + t) * p.part_pitch + s.n0 + n;
#pragma unroll
        for (int r = 0; r < kRun; r += 4) *reinterpret_cast<v4i*>(out + r) = sum[a + r / 4][b];  // (rows are padded to whole runs)
      }
    } else {
      float sb[kRun], bias[kRun];
#pragma unroll
      for (int r = 0; r < kRun; ++r) {
        sb[r] = p.b_scale != nullptr ? factors[n + r] : 1.f;
        bias[r] = factors[K::kChannels + n + r];
      }
      each_of<TN, 1>([&](auto of) {
        constexpr int b = of;
        const uint32_t t = t_in + b * 16;
        if (!full && t >= s.tokens) return;
        float y[kRun];
#pragma unroll
        for (int r = 0; r < kRun; ++r) y[r] = scaled((float)sum[a + r / 4][b][r % 4], sa[b], sb[r], bias[r]);
        if (END == kTail) {
          float x[kRun];
          if (full || kClamped) {
#pragma unroll
            for (int r = 0; r < kRun; ++r) x[r] = p.drop.relu ? (float)ahead[b][r] : 1.f;
            if (p.drop.relu && a + K::kTilesOfRun < CN) fetch(b, n_in + K::channel_row(a + K::kTilesOfRun, 0));
          } else {
            load_gate<T, kRun>(x, p, w[b], row[b], s.n0 + n, left);
          }
          tail_n<kRun>(y, x, p, w[b], row[b], s.n0 + n);
        }
        store_n_within<T, kRun>(static_cast<T*>(p.y.p) + s.m * p.y.pitch + (s.t0 + t) * p.y.ld + s.n0 + n, left, y);
      });
    }
  });
}

template <typename T, int END, int CN, int TN, int CW, int TW, int SLOTS>
__global__ void __launch_bounds__(CW* TW* kWave) product_tile_kernel(Task p) {
  using K = TileKernel<T, CN, TN, CW, TW, SLOTS>;
  __shared__ __align__(1024) char lds[K::kLdsBytes];
  const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), cw = wave % CW, tw = wave / CW;
  const uint32_t across = (uint32_t)((p.channels + K::kChannels - 1) / K::kChannels);
  const uint32_t down = (uint32_t)((p.rows + K::kTokens - 1) / K::kTokens);
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);

  // The tiles of this workgroup: its die's run, in the order of the workgroups there.
  const Run run = run_of(blockIdx.x, gridDim.x, across * down * p.workers * p.splits);

  // What is asked for: number j of a wavefront's loads takes 8 rows of the channels' or the tokens', a row eight lanes.
  uint64_t base_b, base_a;
  uint32_t bytes_b, bytes_a, offset[K::kLoads];
  auto load_one = [&](int j, uint32_t slot) {
    const bool of_b = j < K::kLoadsOfB;
    load_to_lds(of_b ? base_b : base_a, of_b ? bytes_b : bytes_a, offset[j], lds0 + slot + (j * K::kWaves + wave) * 8 * kDepth);
  };
  // After a stage's loads: the next stage's.  Past the last one every address is out of bounds: nothing is read, and what the loads clear
  // is not looked at; they keep the count of a stage's loads.
  int ahead;  // stages not asked for, negative past the last
  auto asked_one = [&]() {
    --ahead;
    base_b += kDepth;
    base_a += kDepth;
    bytes_b = ahead > 0 ? bytes_b - kDepth : 0u;
    bytes_a = ahead > 0 ? bytes_a - kDepth : 0u;
  };
  auto after = [](uint32_t slot) { return slot + K::kStageBytes == K::kRing ? 0u : slot + K::kStageBytes; };
  // A tile's first stages, and its factors.
  auto begin = [&](const Spot& s, uint32_t parity) {
    const uint64_t k = s.split * p.split_depth;
    base_b = reinterpret_cast<uint64_t>(p.b.p) + s.m * p.b.pitch + s.n0 * p.b.ld + k;
    base_a = reinterpret_cast<uint64_t>(p.a.p) + s.m * p.a.pitch + s.t0 * p.a.ld + k;
    bytes_b = (s.channels - 1) * (uint32_t)p.b.ld + (s.depth + 15u) / 16u * 16u;
    bytes_a = (s.tokens - 1) * (uint32_t)p.a.ld + (s.depth + 15u) / 16u * 16u;
#pragma unroll
    for (int j = 0; j < K::kLoads; ++j) {
      const bool of_b = j < K::kLoadsOfB;
      const uint32_t r = ((of_b ? j : j - K::kLoadsOfB) * K::kWaves + wave) * 8 + lane / 8;
      const uint32_t c = lane % 8 ^ (of_b ? moved_by<K::kWide>(r) : moved_by<false>(r));
      offset[j] = min(r, (of_b ? s.channels : s.tokens) - 1) * (uint32_t)(of_b ? p.b.ld : p.a.ld) + c * 16;
    }
    ahead = (int)((s.depth + kDepth - 1) / kDepth);
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
#pragma unroll
      for (int j = 0; j < K::kLoads; ++j) load_one(j, k * K::kStageBytes);
      asked_one();
    }
    if (END != kParts) {  // (a vector that is not there has no bytes)
      const uint32_t to = lds0 + K::kRing + parity * K::kFactorBytes;
      for (uint32_t c = wave * kWave; c < 2 * K::kChannels + K::kTokens; c += K::kWaves * kWave) {
        const bool of_b = c < K::kChannels, of_bias = !of_b && c < 2 * K::kChannels;
        const float* from = of_b ? p.b_scale : of_bias ? p.bias : p.a_scale;
        const uint64_t first = of_b ? s.m * p.b_scale_pitch + s.n0 : of_bias ? s.n0 : s.m * p.rows + s.t0;
        const uint32_t at = c - (of_b ? 0 : of_bias ? K::kChannels : 2 * K::kChannels);
        load_words_to_lds(reinterpret_cast<uint64_t>(from + first), from == nullptr ? 0u : (of_b || of_bias ? s.channels : s.tokens) * 4,
                          (at + lane) * 4, to + c * 4);
      }
    }
  };

  // Where a lane reads its rows' codes: an address for each operand and half, and constants for the tiles.
  const uint32_t i = lane % 16, row_c = K::channel_row(0, i);
  const uint32_t at_c = (cw * CN * 16 + row_c) * kDepth + (lane / 16 ^ moved_by<K::kWide>(row_c)) * 16;
  const uint32_t at_t = (K::kChannels + tw * TN * 16 + i) * kDepth + (lane / 16 ^ moved_by<false>(i)) * 16;

  v4i sum[CN][TN], fc[CN], ft[2][TN];
  auto read_c = [&](int g, uint32_t stage) {
    fc[g % CN] = *reinterpret_cast<const v4i*>(lds + stage + (at_c ^ (g / CN * 64u)) + K::channel_row(g % CN, 0) * kDepth);
  };
  auto read_t = [&](int half, int b, uint32_t stage) {
    ft[half][b] = *reinterpret_cast<const v4i*>(lds + stage + (at_t ^ (half * 64u)) + b * 16 * kDepth);
  };
  // Group g: the matrix instructions of channel tile g % CN in half g / CN, and what is read meanwhile, from kMeet on at `next`.
  auto group = [&](int g, uint32_t stage, uint32_t next, bool first, bool last) {
    if (g < K::kMeet) {
      read_c(g + K::kAhead, stage);
    } else if (!last) {
      read_c(g - K::kMeet, next);
    }
    if (g >= K::kOther && g < K::kOther + TN) read_t(1, g - K::kOther, stage);
    if (g >= K::kMeet && !last) {
#pragma unroll
      for (int b = 0; b < TN; ++b)
        if (b * K::kAhead / TN == g - K::kMeet) read_t(0, b, next);
    }
#pragma unroll
    for (int b = 0; b < TN; ++b)
      sum[g % CN][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fc[g % CN], ft[g / CN][b], first && g < CN ? v4i{0, 0, 0, 0} : sum[g % CN][b], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // What lies past the end of the last stage counts as 0 (of one side, that is enough).
  auto cut = [&](int half, int left) {
#pragma unroll
    for (int b = 0; b < TN; ++b) ft[half][b] = before(ft[half][b], half * 64 + (int)(lane / 16) * 16, left);
  };

  uint32_t tile = run.first, parity = 0;
  if (tile >= run.end) return;
  Spot s = spot_of<K>(p, tile, across, down);
  begin(s, 0);
  // The first tile waits for its first stage only (what is asked for behind the stages makes it wait for a little more); large tiles have no
  // registers for a second kind of wait.  48 x 8192 x 8192 18.8 -> 18.1 us.
  constexpr bool kShortWait = CN <= 4;
  if (kShortWait) wait_and_meet<(SLOTS - 1) * K::kLoads>();
  for (;;) {
    const uint32_t stages = (s.depth + kDepth - 1) / kDepth;
    const int left = (int)(s.depth - (stages - 1) * kDepth);
    const bool ragged = left < kDepth;
    if (!kShortWait) wait_and_meet<0>();
    uint32_t slot = 0;
#pragma unroll
    for (int b = 0; b < TN; ++b) read_t(0, b, 0);
#pragma unroll
    for (int g = 0; g < K::kAhead; ++g) read_c(g, 0);
    if (ragged && stages == 1) cut(0, left);
#pragma unroll
    for (int g = 0; g < K::kMeet; ++g) {
      if (g == CN && ragged && stages == 1) cut(1, left);
      group(g, 0, 0, true, false);
    }
    for (uint32_t k = 0; k + 1 < stages; ++k) {
      const uint32_t next = after(slot);
      wait_and_meet<(SLOTS - 2) * K::kLoads>();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < K::kGroups; ++n) {
        const int g = (K::kMeet + n) % K::kGroups;
#pragma unroll
        for (int j = n * K::kAsks; j < (n + 1) * K::kAsks && j < K::kLoads; ++j) load_one(j, slot);
        if (g == 0 && ragged && k + 2 == stages) cut(0, left);
        if (g == CN && ragged && k + 2 == stages) cut(1, left);
        if (g >= K::kMeet)
          group(g, slot, next, false, false);
        else
          group(g, next, 0, false, false);
      }
      asked_one();
      slot = next;
    }
#pragma unroll
    for (int g = K::kMeet; g < K::kGroups; ++g) group(g, 0, 0, false, true);
    wait_and_meet<0>();  // (the loads that found nothing are done, and the stages are read everywhere)

    const Spot done = s;
    tile += run.step;
    const bool more = tile < run.end;
    if (more) {
      s = spot_of<K>(p, tile, across, down);
      begin(s, parity ^ 1u);
    }
    write_tile<K, T, END, CN, TN>(p, done, sum, cw, tw, lane, reinterpret_cast<const float*>(lds + K::kRing + parity * K::kFactorBytes));
    if (!more) break;
    parity ^= 1u;
    if (kShortWait) wait_and_meet<0>();
  }
}

// ---- Few rows of a: the codes of b pass once, and that is the time (1 x 8192 x 8192 12.7 us, 5.3 TB/s; 1 x 4096 x 4096 4.3).
//
// A workgroup makes all tokens' results of CN x 16 channels; its eight wavefronts take 128 codes of depth each in turn (so that together
// they read whole runs of a row) straight into registers, and their sums meet in LDS.  A lane takes 32 bytes of a row, the operands
// of two matrix instructions: which codes meet in one of them does not matter as long as it is the same ones of both sides.
constexpr int kFewWaves = 8, kFewRows = 64, kFewStep = 128;
constexpr uint64_t kFewDepth = 16384, kFewCodes = 3 << 16;

template <typename T, int CN, int TN>
__global__ void __launch_bounds__(kFewWaves* kWave) product_few_kernel(Task p) {
  constexpr int kResults = CN * TN * 256;
  __shared__ __align__(16) int32_t sums[kFewWaves][kResults];
  const uint32_t m = blockIdx.y, lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane % 16;
  const uint64_t n0 = (uint64_t)blockIdx.x * (CN * 16);
  const uint32_t from = lane / 16 * 32, depth = (uint32_t)p.depth;
  const int8_t *b[CN], *a[TN];
#pragma unroll
  for (int c = 0; c < CN; ++c) b[c] = static_cast<const int8_t*>(p.b.p) + m * p.b.pitch + min(n0 + c * 16 + i, p.channels - 1) * p.b.ld + from;
#pragma unroll
  for (int t = 0; t < TN; ++t) a[t] = static_cast<const int8_t*>(p.a.p) + m * p.a.pitch + min((uint64_t)t * 16 + i, p.rows - 1) * p.a.ld + from;
  v4i sum[CN][TN] = {};
  // kMany steps' loads are under way at a time.
  constexpr uint32_t kStride = kFewWaves * kFewStep;
  constexpr int kMany = TN == 1 ? 4 : 2;  // (more with several tiles of tokens takes the registers of a second workgroup: 22.7 us become 24.2 at 48 x 8192 x 8192)
  uint32_t k = wave * kFewStep;
  const uint32_t whole = depth / kFewStep;
  uint32_t steps = whole > wave ? (whole - wave + kFewWaves - 1) / kFewWaves : 0u;
  auto some = [&](auto many) {
    v4i fb[many][CN][2], fa[many][TN][2];
#pragma unroll
    for (int u = 0; u < many; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < CN; ++c) fb[u][c][h] = *(reinterpret_cast<GlobalPtr<v4i>>((GlobalPtr<int8_t>)(b[c] + k + u * kStride)) + h);
#pragma unroll
        for (int t = 0; t < TN; ++t) fa[u][t][h] = *(reinterpret_cast<GlobalPtr<v4i>>((GlobalPtr<int8_t>)(a[t] + k + u * kStride)) + h);
      }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < many; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < CN; ++c)
#pragma unroll
          for (int t = 0; t < TN; ++t) sum[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][c][h], fa[u][t][h], sum[c][t], 0, 0, 0);
    k += many * kStride;
    steps -= many;
  };
  while (steps >= kMany) some(std::integral_constant<int, kMany>{});
  while (steps > 0) some(std::integral_constant<int, 1>{});
  if (k < depth) {  // the row's end: pieces that begin in it are whole in memory, and what is past the end counts as 0 on one side
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = (int)(from + h * 16), left = (int)(depth - k);
      const bool in = at < left;
      v4i fa[TN];
#pragma unroll
      for (int t = 0; t < TN; ++t) fa[t] = in ? before(*reinterpret_cast<const v4i*>(a[t] + k + h * 16), at, left) : v4i{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < CN; ++c) {
        const v4i fb = in ? *reinterpret_cast<const v4i*>(b[c] + k + h * 16) : v4i{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < TN; ++t) sum[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb, fa[t], sum[c][t], 0, 0, 0);
      }
    }
  }
  // [token][channel] of each wavefront: a lane has four channels of a token
#pragma unroll
  for (int c = 0; c < CN; ++c)
#pragma unroll
    for (int t = 0; t < TN; ++t) *reinterpret_cast<v4i*>(&sums[wave][(t * 16 + i) * (CN * 16) + c * 16 + lane / 16 * 4]) = sum[c][t];
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < kResults; e += kFewWaves * kWave) {
    const uint64_t t = e / (CN * 16), n = n0 + e % (CN * 16);
    if (t >= p.rows || n >= p.channels) continue;
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) all += sums[w][e];
    finish<T>((float)all, p, m, t, n);
  }
}

// ---- Few rows that are not coded yet: every workgroup codes them itself, into LDS, while its first codes of b are on their way, and the
// second launch with its rows of codes in between is saved.  The eight wavefronts share the rows: 8 / `spread` of them each.
constexpr int kCodedRows = 4;
constexpr uint32_t kCodedBytes = 40 * 1024;  // of the codes in LDS

inline uint32_t coded_pitch(uint64_t depth) { return (uint32_t)((depth + kFewStep - 1) / kFewStep * kFewStep + 16); }  // 16 rows, 64 banks

template <typename T, int CN>
__global__ void __launch_bounds__(kFewWaves* kWave) product_coded_kernel(Task p, View x, uint32_t spread, uint32_t pitch) {
  constexpr int kMany = 4;
  constexpr uint32_t kStride = kFewWaves * kFewStep;
  __shared__ __align__(16) int32_t sums[kFewWaves][CN * 256];
  __shared__ uint32_t tops[kFewWaves];
  extern __shared__ __align__(16) int8_t codes[];  // [rows][pitch], 0 behind a row's end
  const uint32_t m = blockIdx.y, lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane % 16;
  const uint64_t n0 = (uint64_t)blockIdx.x * (CN * 16);
  const uint32_t from = lane / 16 * 32, depth = (uint32_t)p.depth, rows = (uint32_t)p.rows;
  const int8_t* b[CN];
#pragma unroll
  for (int c = 0; c < CN; ++c) b[c] = static_cast<const int8_t*>(p.b.p) + m * p.b.pitch + min(n0 + c * 16 + i, p.channels - 1) * p.b.ld + from;
  uint32_t k = wave * kFewStep;
  const uint32_t whole = depth / kFewStep;
  uint32_t steps = whole > wave ? (whole - wave + kFewWaves - 1) / kFewWaves : 0u;
  v4i fb[kMany][CN][2];
  auto ask = [&](uint32_t many) {  // (past the last whole step: the last again, which is not used)
#pragma unroll
    for (uint32_t u = 0; u < kMany; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < CN; ++c)
          fb[u][c][h] = *(reinterpret_cast<GlobalPtr<v4i>>((GlobalPtr<int8_t>)(b[c] + k + min(u, many - 1) * kStride)) + h);
  };
  if (steps > 0) ask(min(steps, (uint32_t)kMany));

  // the codes
  const uint32_t row = wave / spread, part = wave % spread, jump = spread * kWave * 8;
  const bool has = row < rows;
  const T* from_x = static_cast<const T*>(x.p) + m * x.pitch + min(row, rows - 1) * x.ld;
  uint32_t top = 0u;
  float v[8];
  for (uint32_t c = (part * kWave + lane) * 8; c < depth; c += jump) {
    load_n<T, 8>(from_x + min(c, depth - 8), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, magnitude_bits(v[e]));
  }
  top = wave_max_bits(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  for (uint32_t w = 0; w < spread; ++w) top = max(top, tops[row * spread + w]);
  const float inv = code_inverse(top);
  const bool once = depth <= jump;  // (a lane's only values are those that it still has)
  if (has) {
    for (uint32_t c = (part * kWave + lane) * 8; c < depth; c += jump) {
      const uint32_t at = min(c, depth - 8);
      if (!once) load_n<T, 8>(from_x + at, v);
      typedef uint32_t two __attribute__((ext_vector_type(2), aligned(1)));
      uint32_t q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = code_nearest(v[e], inv);
      *reinterpret_cast<two*>(codes + row * pitch + at) = two{pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7])};
    }
    if (part == 0)
      for (uint32_t c = depth + lane; c < pitch; c += kWave) codes[row * pitch + c] = 0;
  }
  __syncthreads();

  const int8_t* a = codes + min(i, rows - 1) * pitch + from;
  v4i sum[CN] = {};
  while (steps > 0) {
    const uint32_t many = min(steps, (uint32_t)kMany);
#pragma unroll
    for (uint32_t u = 0; u < kMany; ++u)
      if (u < many) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const v4i fa = *reinterpret_cast<const v4i*>(a + k + u * kStride + h * 16);
#pragma unroll
          for (int c = 0; c < CN; ++c) sum[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][c][h], fa, sum[c], 0, 0, 0);
        }
      }
    k += many * kStride;
    steps -= many;
    if (steps > 0) ask(min(steps, (uint32_t)kMany));
  }
  if (k < depth) {  // a row's end: its last piece is whole in memory, and meets zeros
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = from + h * 16 < depth - k;
      const v4i fa = *reinterpret_cast<const v4i*>(a + k + h * 16);
#pragma unroll
      for (int c = 0; c < CN; ++c) {
        const v4i last = in ? *reinterpret_cast<const v4i*>(b[c] + k + h * 16) : v4i{0, 0, 0, 0};
        sum[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(last, fa, sum[c], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CN; ++c) *reinterpret_cast<v4i*>(&sums[wave][i * (CN * 16) + c * 16 + lane / 16 * 4]) = sum[c];
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < rows * (CN * 16); e += kFewWaves * kWave) {
    const uint32_t t = e / (CN * 16);
    const uint64_t n = n0 + e % (CN * 16);
    if (n >= p.channels) continue;
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) all += sums[w][e];
    uint32_t r = 0u;
    for (uint32_t w = 0; w < spread; ++w) r = max(r, tops[t * spread + w]);
    const float sb = p.b_scale != nullptr ? p.b_scale[m * p.b_scale_pitch + n] : 1.f;
    const float bias = p.bias != nullptr ? p.bias[n] : 0.f;
    static_cast<T*>(p.y.p)[m * p.y.pitch + t * p.y.ld + n] = (T)scaled((float)all, code_step(r), sb, bias);
  }
}

// The splits' sums joined, four channels a lane: a launch's latency and their bytes (48 x 8192 4 us).
template <typename T>
__global__ void __launch_bounds__(kBlock) product_join_kernel(Task p) {
  const uint32_t m = blockIdx.y, each = p.part_pitch / 4;
  const uint64_t index = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
  const uint64_t t = index / each;
  if (t >= p.rows) return;
  const uint32_t n = (uint32_t)(index - t * each) * 4;
  int64_t sum[4] = {0, 0, 0, 0};
  for (uint32_t s = 0; s < p.splits; ++s) {
    const v4i v = *reinterpret_cast<const v4i*>(p.parts + (((uint64_t)s * p.workers + m) * p.rows + t) * p.part_pitch + n);
#pragma unroll
    for (int r = 0; r < 4; ++r) sum[r] += v[r];
  }
  const uint64_t left = n < p.channels ? p.channels - n : 0;
  if (left == 0) return;
  float sb[4] = {1.f, 1.f, 1.f, 1.f}, bias[4] = {0.f, 0.f, 0.f, 0.f}, y[4];
  const float sa = p.a_scale != nullptr ? p.a_scale[m * p.rows + t] : 1.f;
  if (p.b_scale != nullptr) load_n_within<float, 4>(p.b_scale + m * p.b_scale_pitch + n, left, 0.f, sb);
  if (p.bias != nullptr) load_n_within<float, 4>(p.bias + n, left, 0.f, bias);
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = scaled((float)sum[r], sa, sb[r], bias[r]);
  if (p.drops) {
    float x[4];
    uint32_t row = (uint32_t)t;
    const uint32_t w = worker_of(p, m, &row);
    load_gate<T, 4>(x, p, w, row, n, left);
    tail_n<4>(y, x, p, w, row, n);
  }
  store_n_within<T, 4>(static_cast<T*>(p.y.p) + m * p.y.pitch + t * p.y.ld + n, left, y);
}

// Whether every row's pieces of 16 codes are 16-byte aligned and a tile's rows lie within 32 bits of each other.
bool pieces_aligned(const Product& p) {
  auto fits = [](const View& v) {
    return reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.ld % 16 == 0 && v.pitch % 16 == 0 && v.ld < (1u << 23);
  };
  return fits(p.a) && fits(p.b);
}

enum class Way { kAny, kFew, kFlatTiles, kNarrowTiles, kSmallTiles, kLargeTiles };

struct Plan {
  Way way;
  uint32_t splits;
  uint64_t split_depth;
};

uint64_t over(uint64_t n, uint64_t by) { return (n + by - 1) / by; }

uint64_t part_pitch(const Product& p) { return over(p.channels, 8) * 8; }  // (rows of partial sums hold whole runs)

// Which tiles, and how many splits of the depth.  Estimated, in us, from what was measured: a stage takes a fixed time where few CUs work (the
// loads' latency) and more where all do; each tile of a workgroup has its time beside its stages (first loads, scaling, writing); joining splits
// takes 5 and their bytes at 4 TB/s.  All sides, us, tokens x channels x depth, narrow (64 channels x 128 tokens) / small (128 x 128) / large tiles (256 x 256): 333 x 1003 x 1000 6.9 / 8.7 / 12; 200 x 8192 x 5000 22.7 / 26 / 58;
// 1024 x 1024 x 8192 24.4 / 31.7 / 75; 2048 x 2048 x 2048 18.6 / 14.7 / 26.7; 8192 x 8192 x 1024 166 / 134 / 94; 8192 x 8192 x 8192 - / 585 /
// 407; one / two splits of the small: 1024 x 1024 x 8192 31 / 25; 4096 x 512 x 4096 19.8 / 24.6.  Flat tiles (128 x 64) against narrow: 64 x 16384 x
// 4096 14.3 / 16.5; 64 x 32768 x 512 5.7 / 6.6; 129 x 8192 x 8192 23.5 / 27.1.
void by_tiles(const Product& p, Plan* plan) {
  struct Kind {
    Way way;
    uint64_t tokens, channels;
    double stage, busy_stage, tile;
  };
  constexpr Kind kinds[] = {{Way::kNarrowTiles, 128, 64, 0.30, 0.17, 3.0}, {Way::kFlatTiles, 64, 128, 0.30, 0.17, 3.0},
                            {Way::kSmallTiles, 128, 128, 0.43, 0.19, 3.0}, {Way::kLargeTiles, 256, 256, 1.2, 0.4, 8.0}};
  constexpr double kCus = 256.0;
  const uint32_t least = plan->splits;  // that keep the sums inside 32 bits
  double best = 0.0;
  for (const Kind& kind : kinds) {
    const uint64_t tiles = over(p.rows, kind.tokens) * over(p.channels, kind.channels) * p.workers;
    for (uint32_t splits = least; splits <= std::max(least, 8u); ++splits) {
      const uint64_t stages = over(over(p.depth, kDepth), splits), all = tiles * splits;
      if (splits > least && (all > (uint64_t)kCus || stages < 8)) break;
      const double stage = kind.stage + kind.busy_stage * std::min(1.0, (double)all / kCus);
      double us = std::ceil((double)all / kCus) * ((double)stages * stage + kind.tile);
      if (splits > 1) us += 5.0 + (double)(splits * p.workers * p.rows) * (double)part_pitch(p) * 8e-6 / 4.0;
      if (best == 0.0 || us < best) {
        best = us;
        plan->way = kind.way;
        plan->splits = splits;
      }
    }
  }
}

// The kernel for few rows takes time with its rows and the depth, tiles hardly with the rows.  Measured, us, few / tiles, rows x channels x depth:
// 1 x 4096 x 16384 15.4 / 18.9; 16 x 512 x 8192 8.9 / 10.2; 16 x 512 x 16384 15.9 / 12.3; 48 x 8192 x 4096 12.3 / 12.9; 64 x 4096 x 1024
// 4.9 / 6.0; 64 x 512 x 4096 11.1 / 9.2; 32 x 8192 x 8192 17.9 / 18.3; 48 x 8192 x 8192 21.3 / 19.1; 32 x 16384 x 4096 17.5 / 13.5; 16 x
// 16384 x 4096 13.6 / 13.1.
bool few_is_sooner(const Product& p) {
  const uint64_t groups = over(p.channels, 16) * p.workers;
  return p.rows <= kFewRows && p.depth <= kFewDepth && p.rows * p.depth <= kFewCodes && (p.rows <= 16 || groups <= (p.rows <= 48 ? 512 : 256));
}

Plan plan_of(const Product& p) {
  Plan plan{};
  plan.splits = (uint32_t)std::max<uint64_t>(over(p.depth, kMaxDepth), 1);
  if (!pieces_aligned(p) || p.depth == 0) {
    plan.way = Way::kAny;
  } else if (few_is_sooner(p)) {
    plan.way = Way::kFew;
    plan.splits = 1;
  } else {
    by_tiles(p, &plan);
  }
  plan.split_depth = plan.splits == 1 ? p.depth : over(over(p.depth, plan.splits), kDepth) * kDepth;
  if (plan.splits > 1) plan.splits = (uint32_t)over(p.depth, plan.split_depth);  // (no split without any depth)
  return plan;
}

template <typename T, int CN, int TN, int CW, int TW, int SLOTS>
void launch_tiles(const Task& t, hipStream_t s) {
  using K = TileKernel<T, CN, TN, CW, TW, SLOTS>;
  const uint64_t tiles = over(t.rows, K::kTokens) * over(t.channels, K::kChannels) * t.workers * t.splits;
  const dim3 grid((uint32_t)std::min<uint64_t>(tiles, K::kWorkgroups));
  if (t.parts != nullptr) {
    product_tile_kernel<T, kParts, CN, TN, CW, TW, SLOTS><<<grid, K::kThreads, 0, s>>>(t);
  } else if (t.drops) {
    // (float32 results and the tail together take more registers than the large tiles leave)
    if constexpr (sizeof(T) == 4 && CN > 4)
      launch_tiles<T, 4, 2, 2, 4, 2>(t, s);
    else
      product_tile_kernel<T, kTail, CN, TN, CW, TW, SLOTS><<<grid, K::kThreads, 0, s>>>(t);
  } else {
    product_tile_kernel<T, kScaled, CN, TN, CW, TW, SLOTS><<<grid, K::kThreads, 0, s>>>(t);
  }
}

// Codes of a are read again by every workgroup: two tiles of channels each, where that leaves a workgroup for every CU.
// Measured, us, one / two tiles (depth 8192): 1 token, 8192 channels 13.2 / 15.3; 1, 16384 13.4 / 12.3; 16, 8192 17.7 / 14.2; 64, 8192 39.4 / 27.6.
template <typename T, int TN>
void launch_few(const Task& t, hipStream_t s) {
  auto launch = [&](auto tiles) {
    product_few_kernel<T, tiles, TN><<<dim3((uint32_t)over(t.channels, tiles * 16), t.workers), kFewWaves * kWave, 0, s>>>(t);
  };
  if constexpr (TN <= 3) {  // (more rows: few_is_sooner has less channels)
    if (over(t.channels, 32) * t.workers >= (t.rows > 4 ? 256 : 512)) return launch(std::integral_constant<int, 2>{});
  }
  launch(std::integral_constant<int, 1>{});
}

Task task_of(const Product& p) {
  Task t{};
  t.workers = p.workers;
  t.rows_of_worker = (uint32_t)p.rows_of_worker;
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
  if (p.drop != nullptr) {
    t.drop = *p.drop;
    t.drops = 1;
  }
  return t;
}

template <typename T>
hipError_t product_typed(const Product& p, void* scratch, hipStream_t s) {
  const Plan plan = plan_of(p);
  Task t = task_of(p);
  t.split_depth = plan.split_depth;
  t.splits = plan.splits;
  t.part_pitch = (uint32_t)part_pitch(p);
  t.parts = plan.splits > 1 ? static_cast<int32_t*>(scratch) : nullptr;
  switch (plan.way) {
    case Way::kFew:
      if (p.rows <= 16)
        launch_few<T, 1>(t, s);
      else if (p.rows <= 32)
        launch_few<T, 2>(t, s);
      else if (p.rows <= 48)
        launch_few<T, 3>(t, s);
      else
        launch_few<T, 4>(t, s);
      break;
    case Way::kFlatTiles: launch_tiles<T, 2, 2, 4, 2, 4>(t, s); break;
    case Way::kNarrowTiles: launch_tiles<T, 2, 2, 2, 4, 4>(t, s); break;
    case Way::kSmallTiles:
      // More tiles than CUs: two stages each and two workgroups a CU, one writes while the other multiplies (8 x 1024 x 1024 x 512 16.8 -> 14.0 us);
      // else four stages (1537 x 2053 x 1999 19.0 -> 16.6).
      if (over(p.rows, 128) * over(p.channels, 128) * p.workers * plan.splits > 256)
        launch_tiles<T, 4, 2, 2, 4, 2>(t, s);
      else
        launch_tiles<T, 4, 2, 2, 4, 4>(t, s);
      break;
    case Way::kLargeTiles:
      launch_tiles<T, 8, 4, 2, 4, 2>(t, s);
      break;
    default: {
      const uint64_t tiles = over(p.rows, kAnyTile) * over(p.channels, kAnyTile);
      product_any_kernel<T><<<dim3((uint32_t)tiles, p.workers, plan.splits), kBlock, 0, s>>>(t);
    }
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess || plan.splits == 1) return e;
  product_join_kernel<T><<<dim3((uint32_t)over(p.rows * (t.part_pitch / 4), kBlock), p.workers), kBlock, 0, s>>>(t);
  return hipGetLastError();
}

// The rows of all workers as those of one, where they lie so and b is the same.
Product joined(Product p) {
  p.rows_of_worker = p.rows;
  if (p.workers > 1 && p.b.pitch == 0 && p.b_scale_pitch == 0 && p.a.pitch == p.rows * p.a.ld && p.y.pitch == p.rows * p.y.ld) {
    p.rows *= p.workers;
    p.workers = 1;
    p.a.pitch = p.y.pitch = 0;
  }
  return p;
}

// x in the place of a, all workers' rows together where they share b.
Product coded_rows(const Product& p, const View& x) {
  Product c = p;
  c.a = x;
  return joined(c);
}

}  // namespace

size_t product_scratch_bytes(const Product& given) {
  const Product p = joined(given);
  const Plan plan = plan_of(p);
  return plan.splits > 1 ? plan.splits * (size_t)p.workers * p.rows * part_pitch(p) * sizeof(int32_t) : 0;
}

hipError_t launch_product(const Product& given, void* scratch, hipStream_t s) {
  const Product p = joined(given);
  switch (p.type) {
    case TNG_TYPE_F32: return product_typed<float>(p, scratch, s);
    case TNG_TYPE_BF16: return product_typed<bf16_t>(p, scratch, s);
    default: return product_typed<f16_t>(p, scratch, s);
  }
}

// Every workgroup reads and codes the rows again, so few of both.  Measured, us, with / without (a launch to code, a launch of
// product_few_kernel), bfloat16: 1 row 4096 -> 4096 5.1 / 6.8, 4096 -> 16384 14.0 / 14.4, 8192 -> 8192 14.7 / 15.7; 4 rows 7.0 / 7.7,
// 16.4 / 14.9, 18.6 / 16.6; 8 rows of 4096 -> 4096 9.3 / 8.0.
bool coded_product_applies(const Product& p, const View& x) {
  const Product c = coded_rows(p, x);
  const bool aligned = reinterpret_cast<uintptr_t>(c.b.p) % 16 == 0 && c.b.ld % 16 == 0 && c.b.pitch % 16 == 0 && c.b.ld < (1u << 23);
  const bool shared = c.workers > 1 && c.b.pitch == 0;  // (by rows that do not lie together)
  const bool few = c.rows == 1 || (c.rows <= kCodedRows && c.rows * c.depth <= 16384 && over(c.channels, 16) * c.workers <= 512);
  return aligned && !shared && few && c.depth >= 8 && c.depth <= kMaxDepth && c.rows * coded_pitch(c.depth) <= kCodedBytes;
}

hipError_t launch_coded_product(const Product& given, const View& x, hipStream_t s) {
  const Product p = coded_rows(given, x);
  const Task t = task_of(p);
  uint32_t spread = kFewWaves;
  while (spread * p.rows > kFewWaves) spread /= 2;
  const uint32_t pitch = coded_pitch(p.depth);
  auto launch = [&](auto type, auto tiles) {
    product_coded_kernel<decltype(type), tiles><<<dim3((uint32_t)over(p.channels, tiles * 16), p.workers), kFewWaves * kWave, p.rows * pitch, s>>>(
        t, p.a, spread, pitch);
  };
  auto typed = [&](auto tiles) {
    switch (p.type) {
      case TNG_TYPE_F32: launch(float{}, tiles); break;
      case TNG_TYPE_BF16: launch(bf16_t{}, tiles); break;
      default: launch(f16_t{}, tiles);
    }
  };
  if (over(p.channels, 32) * p.workers >= 512)  // (as launch_few)
    typed(std::integral_constant<int, 2>{});
  else
    typed(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

}  // namespace tng
