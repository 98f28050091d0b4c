// Embedding tables: rows by tokens, and the gradient of the table from tokens in sorted order (gfx950).
#include "tng_layer_device.hpp"

#include <algorithm>
#include <type_traits>

namespace tng {
namespace {

template <typename T>
using Vec8 = T __attribute__((ext_vector_type(8), aligned(alignof(T))));

// The row of the table that a token asks for, or `rows` where it is outside of it.
template <typename I>
__device__ __forceinline__ uint32_t row_of(const I* ids, uint64_t at, uint64_t rows) {
  const int64_t id = (int64_t)ids[at];
  return id >= 0 && (uint64_t)id < rows ? (uint32_t)id : (uint32_t)rows;
}

// Results of more bytes are written past the caches: the memory-side cache, of 256 MiB, does not hold them beside what is read.
constexpr uint64_t kPast = 128u << 20;

struct EmbedTask {
  uint64_t rows, cols, eights;  // tokens of a worker; columns; lanes that a row takes
  uint64_t vocabulary;
  View ids, table, y;
  float scale;
  bool past;  // y is written past the caches
};

// y = scale table[id].  What it moves bounds it: 32768 tokens of 4096 bfloat16, whose 15000 rows and result are 390 MB, 74 us; 3 x 20011 of 1003, float32 to
// float16, rows at odd places, half of them of no token, 38 us, of tokens all 51, in which 240 MB come out of the caches.  A lane takes eight columns of kMany
// tokens' rows (the row's last eight where it ends inside them: what two lanes write of one column is the same), so that their tokens, and then their rows, are
// on the way together.
template <typename I, typename W, typename T, bool NARROW>
__global__ void __launch_bounds__(kBlock) embed_kernel(EmbedTask p) {
  constexpr int kMany = 4;
  const uint32_t m = blockIdx.y;
  const I* ids = static_cast<const I*>(p.ids.p) + m * p.ids.pitch;
  const W* table = static_cast<const W*>(p.table.p) + m * p.table.pitch;
  T* y = static_cast<T*>(p.y.p) + m * p.y.pitch;
  const uint64_t n = p.rows * p.eights, first = (uint64_t)blockIdx.x * (kBlock * kMany) + threadIdx.x;
  uint64_t t[kMany], c[kMany];
  uint32_t row[kMany];
#pragma unroll
  for (int k = 0; k < kMany; ++k) {
    const uint64_t at = min(first + k * kBlock, n - 1);
    t[k] = (uint32_t)at / (uint32_t)p.eights;  // (no matrix has 2^32 eights, and 64 bits take four times the instructions)
    c[k] = (at - t[k] * p.eights) * 8;
    if (!NARROW) c[k] = min(c[k], p.cols - 8);
    row[k] = row_of<I>(ids, t[k] * p.ids.ld, p.vocabulary);
  }
  Vec8<W> w[kMany];
#pragma unroll
  for (int k = 0; k < kMany; ++k) {
    w[k] = Vec8<W>{};
    if (row[k] >= p.vocabulary) continue;
    const W* from = table + (uint64_t)row[k] * p.table.ld + c[k];
    if (NARROW) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) w[k][i] = i < p.cols ? from[i] : (W)0.f;
    } else {
      w[k] = *reinterpret_cast<GlobalPtr<Vec8<W>>>((GlobalPtr<W>)from);
    }
  }
#pragma unroll
  for (int k = 0; k < kMany; ++k) {
    if (first + k * kBlock >= n) continue;
    Vec8<T> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)(row[k] < p.vocabulary ? pinned((float)w[k][i] * p.scale) : 0.f);
    T* to = y + t[k] * p.y.ld + c[k];
    if (NARROW) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i)
        if (i < p.cols) to[i] = v[i];
    } else if (p.past) {
      __builtin_nontemporal_store(v, reinterpret_cast<Vec8<T>*>(to));
    } else {
      *reinterpret_cast<Vec8<T>*>(to) = v;
    }
  }
}

// No row to read: all tokens are outside.
template <typename T>
__global__ void __launch_bounds__(kBlock) embed_nothing_kernel(uint64_t rows, uint64_t cols, View y) {
  const uint64_t e = block_number() * kBlock + threadIdx.x;
  if (e >= rows * cols) return;
  const uint64_t r = e / cols;
  static_cast<T*>(y.p)[blockIdx.z * y.pitch + r * y.ld + (e - r * cols)] = (T)0.f;
}

template <typename I, typename W, typename T>
void embed_typed(uint32_t workers, EmbedTask& p, hipStream_t s) {
  if (p.vocabulary == 0) {
    embed_nothing_kernel<T><<<grid_of((p.rows * p.cols + kBlock - 1) / kBlock, workers), kBlock, 0, s>>>(p.rows, p.cols, p.y);
    return;
  }
  p.eights = (p.cols + 7) / 8;
  const dim3 grid((uint32_t)((p.rows * p.eights + kBlock * 4 - 1) / (kBlock * 4)), workers);
  if (p.cols < 8)
    embed_kernel<I, W, T, true><<<grid, kBlock, 0, s>>>(p);
  else
    embed_kernel<I, W, T, false><<<grid, kBlock, 0, s>>>(p);
}

template <typename I, typename W>
void embed_to(tng_type type, uint32_t workers, EmbedTask& p, hipStream_t s) {
  switch (type) {
    case TNG_TYPE_F32: embed_typed<I, W, float>(workers, p, s); break;
    case TNG_TYPE_BF16: embed_typed<I, W, bf16_t>(workers, p, s); break;
    default: embed_typed<I, W, f16_t>(workers, p, s); break;
  }
}

template <typename I>
void embed_from(tng_type table, tng_type type, uint32_t workers, EmbedTask& p, hipStream_t s) {
  switch (table) {
    case TNG_TYPE_F32: embed_to<I, float>(type, workers, p, s); break;
    case TNG_TYPE_BF16: embed_to<I, bf16_t>(type, workers, p, s); break;
    default: embed_to<I, f16_t>(type, workers, p, s); break;
  }
}

// ---- the gradient of the table
//
// A row's gradient is the sum of its tokens' rows of dy.  Tokens are sorted, kSorted at a time, by a workgroup each, in LDS: the tokens of a row lie
// together then, a run, in the order that they came in, whatever ran first.  Sums are taken in that order.  Runs that cross the ends of pieces of kPiece sorted
// places are summed by pieces first, and those that cross the ends of kPiece pieces by such wholes: whatever tokens come, no sum is a long chain, and
// each row of dy is read once.  Every row of the table is written, those of no token with zeros.
constexpr uint32_t kSorted = 4096, kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr uint32_t kFew = kBlock;                           // so many a workgroup picks its rows' from, without an order made before
constexpr uint32_t kPiece = 32, kWhole = kPiece * kPiece;  // places of a piece, and of a piece of pieces
constexpr uint32_t kMostBins = 256, kMostEach = 16;

struct EmbedGradTask {
  uint64_t rows, cols, vocabulary;
  View ids, dy, dtable;
  float scale;
  uint32_t bits;          // of a row's number; the largest number they hold stands for no row
  uint32_t blocks;        // of kSorted tokens, of a worker
  uint32_t places;        // of a block that are written: those behind the last token hold no row
  uint32_t each, groups;  // rows of the table that a workgroup writes (kMostEach at most), and how many such groups there are
  uint32_t *row, *token;  // [worker][block][kSorted]: sorted rows, and the token's number
  uint32_t* begin;        // [worker][block][groups + 1]: where a group's rows begin in a block
  float *piece, *whole;   // [worker][block][places / kPiece][2][cols], and / kWhole (or null): of the run that comes in, and of the one that goes out
  bool past;              // dtable is written past the caches
};

// Where each group of rows begins in a block: the first place whose row is no less.
__device__ __forceinline__ void groups_begin(const EmbedGradTask& p, uint32_t m, const uint32_t* keys, uint32_t places) {
  for (uint32_t g = threadIdx.x; g <= p.groups; g += blockDim.x) {
    const uint64_t want = min((uint64_t)g * p.each, p.vocabulary);
    uint32_t low = 0u, high = places;
    while (low < high) {
      const uint32_t mid = (low + high) / 2;
      if (keys[mid] < want)
        low = mid + 1;
      else
        high = mid;
    }
    p.begin[((uint64_t)m * p.blocks + blockIdx.x) * (p.groups + 1) + g] = low;
  }
}

// Least significant digits first, of 2^digit bins.  A wavefront takes consecutive places, 64 at a time: lanes of one digit find each other by ballots, and
// the wavefront's counter of that digit says how many came before them.  That all is one CU's work is what bounds it: six instructions a bit and token for
// the ballots.  2048 tokens of 32000 rows 9.7 us, 4096 of 4099 rows 12 (8192 at a time 18, and the gradient of 30000 tokens into 20000 x 256 43 instead of 36).
template <typename I, int ITEMS>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(EmbedGradTask p, uint32_t digit, uint32_t passes) {
  __shared__ uint32_t keys[ITEMS * kSortThreads];
  __shared__ uint16_t from[ITEMS * kSortThreads];
  __shared__ uint32_t count[kMostBins][kSortWaves + 1];  // (one more: the bins of a wavefront lie in different banks)
  __shared__ uint32_t of_wave[kSortWaves];
  const uint32_t m = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, bins = 1u << digit;
  const uint64_t first = (uint64_t)blockIdx.x * kSorted;
  const I* ids = static_cast<const I*>(p.ids.p) + m * p.ids.pitch;
  const uint32_t none = (1u << p.bits) - 1u, base = wave * (ITEMS * kWave) + lane;
  uint32_t key[ITEMS], at[ITEMS], place[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    at[i] = base + i * kWave;
    const uint32_t r = row_of<I>(ids, min(first + at[i], p.rows - 1) * p.ids.ld, p.vocabulary);
    key[i] = first + at[i] < p.rows && r < p.vocabulary ? r : none;
  }
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t down = pass * digit;
    for (uint32_t c = threadIdx.x; c < bins * (kSortWaves + 1); c += kSortThreads) (&count[0][0])[c] = 0u;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t d = key[i] >> down & (bins - 1u);
      uint64_t same = ~0ull;
      for (uint32_t b = 0; b < digit; ++b) {
        const uint64_t has = __ballot(d >> b & 1u);
        same &= (d >> b & 1u) ? has : ~has;
      }
      const uint32_t before = __popcll(same & ((1ull << lane) - 1ull));
      volatile uint32_t* mine = &count[d][wave];
      const uint32_t so_far = *mine;
      place[i] = so_far + before;
      __builtin_amdgcn_wave_barrier();  // (all have read; a wavefront's accesses to LDS keep their order)
      if (before == 0u) *mine = so_far + (uint32_t)__popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // counters become where a wavefront's places of a digit begin: a lane sums a bin, then the bins of a wavefront, then those before it
    uint32_t sum = 0u;
    if (threadIdx.x < bins) {
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) {
        const uint32_t c = count[threadIdx.x][w];
        count[threadIdx.x][w] = sum;
        sum += c;
      }
    }
    uint32_t upto = sum;
#pragma unroll
    for (uint32_t off = 1; off < kWave; off *= 2) {
      const uint32_t other = __shfl_up(upto, off, kWave);
      if (lane >= off) upto += other;
    }
    if (lane == kWave - 1) of_wave[wave] = upto;
    __syncthreads();
    if (threadIdx.x < bins) {
      upto -= sum;
      for (uint32_t w = 0; w < wave; ++w) upto += of_wave[w];
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) count[threadIdx.x][w] += upto;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t to = count[key[i] >> down & (bins - 1u)][wave] + place[i];
      keys[to] = key[i];
      from[to] = (uint16_t)at[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      key[i] = keys[base + i * kWave];
      at[i] = from[base + i * kWave];
    }
    __syncthreads();
  }
  const uint64_t to = ((uint64_t)m * p.blocks + blockIdx.x) * kSorted;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    p.row[to + base + i * kWave] = key[i];
    p.token[to + base + i * kWave] = (uint32_t)(first + at[i]);
  }
  groups_begin(p, m, keys, ITEMS * kSortThreads);
}

// What a lane has of a row: Q times four columns, LANES fours apart, so that a wavefront's accesses have no gaps.  Where a row ends inside a four, the row's
// last four are taken (what two lanes have of one column is the same).  NARROW: rows of less than four columns.
template <int Q>
struct Columns {
  uint64_t at[Q];
  bool has[Q];
};
template <int LANES, int Q, bool NARROW>
__device__ __forceinline__ Columns<Q> columns_of(uint32_t chunk, uint32_t lane, uint64_t cols) {
  Columns<Q> c;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    c.at[q] = ((uint64_t)chunk * (LANES * Q) + q * LANES + lane) * 4;
    c.has[q] = c.at[q] < cols;
    c.at[q] = NARROW ? 0 : min(c.at[q], cols - 4);
  }
  return c;
}

template <typename T, int Q, bool NARROW>
struct Some {
  typedef T vec __attribute__((ext_vector_type(4), aligned(alignof(T))));
  vec v[Q];
  __device__ __forceinline__ void load(const T* row, const Columns<Q>& c, uint64_t cols) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (NARROW) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) v[q][i] = i < cols ? row[i] : (T)0.f;
      } else {
        v[q] = *reinterpret_cast<GlobalPtr<vec>>((GlobalPtr<T>)(row + c.at[q]));
      }
    }
  }
  __device__ __forceinline__ void add_to(float (&sum)[Q][4], bool counted) const {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[q][i] += counted ? (float)v[q][i] : 0.f;
  }
};

// Numbers f(0) .. f(count - 1), the same for a wavefront, many on the way at a time; past the end the last one again, which is not counted.
template <int MANY, typename T, int Q, bool NARROW, typename F>
__device__ __forceinline__ void add_many(F row, uint32_t& first, uint32_t count, const Columns<Q>& c, uint64_t cols, float (&sum)[Q][4]) {
  Some<T, Q, NARROW> some[MANY];
#pragma unroll
  for (uint32_t k = 0; k < MANY; ++k) some[k].load(row(min(first + k, count - 1)), c, cols);
#pragma unroll
  for (uint32_t k = 0; k < MANY; ++k) some[k].add_to(sum, first + k < count);
  first += MANY;
}
template <typename T, int Q, bool NARROW, typename F>
__device__ __forceinline__ void add_all(F row, uint32_t count, const Columns<Q>& c, uint64_t cols, float (&sum)[Q][4]) {
  constexpr int kMany = sizeof(T) == 4 ? 8 : 16;
  uint32_t k = 0;
  while (k + kMany / 2 < count) add_many<kMany, T, Q, NARROW>(row, k, count, c, cols, sum);
  while (k < count) add_many<2, T, Q, NARROW>(row, k, count, c, cols, sum);
}

// The rows of dy of the tokens that lanes first .. first + count - 1 hold.
template <typename T, int Q, bool NARROW>
__device__ __forceinline__ void add_tokens(const T* dy, uint64_t ld, uint32_t token, uint32_t first, uint32_t count, const Columns<Q>& c, uint64_t cols,
                                           float (&sum)[Q][4]) {
  add_all<T, Q, NARROW>([&](uint32_t k) { return dy + (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)token, (int)(first + k)) * ld; }, count, c, cols, sum);
}
// Those of places first .. end - 1: a wavefront reads 32 tokens at a time, a lane one.
template <typename T, int Q, bool NARROW>
__device__ __forceinline__ void add_rows(const T* dy, uint64_t ld, const uint32_t* token, uint32_t first, uint32_t end, const Columns<Q>& c, uint64_t cols,
                                         float (&sum)[Q][4]) {
  for (; first < end; first += kPiece) {
    const uint32_t count = min(end - first, kPiece);
    add_tokens<T, Q, NARROW>(dy, ld, token[first + min(threadIdx.x % kPiece, count - 1)], 0, count, c, cols, sum);
  }
}

// Parts that lie `stride` apart.
template <int Q, bool NARROW>
__device__ __forceinline__ void add_parts(const float* part, uint64_t stride, uint32_t count, const Columns<Q>& c, uint64_t cols, float (&sum)[Q][4]) {
  add_all<float, Q, NARROW>([&](uint32_t k) { return part + k * stride; }, count, c, cols, sum);
}

template <int Q, bool NARROW>
__device__ __forceinline__ void store_sum(float* to, const Columns<Q>& c, uint64_t cols, const float (&sum)[Q][4], float scale, bool past) {
  typedef float four __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (!c.has[q]) continue;
    four v;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[i] = sum[q][i] * scale;
    if (NARROW) {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (i < cols) to[i] = v[i];
    } else if (past) {
      __builtin_nontemporal_store(v, reinterpret_cast<four*>(to + c.at[q]));
    } else {
      *reinterpret_cast<four*>(to + c.at[q]) = v;
    }
  }
}

// The two runs that cross the ends of a piece (or of a piece of pieces): the sum of the one that comes in, as far as it goes, and of the one that
// begins here and goes on.  LANES take a piece.  3 x 20011 tokens of 1003 float16, 120 MB, 26 us; few pieces take the latency of their loads, 10.
template <typename T, bool WHOLE, int LANES, int Q, bool NARROW>
__global__ void __launch_bounds__(kBlock) embed_pieces_kernel(EmbedGradTask p) {
  constexpr uint32_t kPlaces = WHOLE ? kWhole : kPiece;
  const uint32_t m = blockIdx.z, each = p.places / kPlaces, lane = threadIdx.x % LANES;
  const uint32_t number = blockIdx.x * (kBlock / LANES) + __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
  if (number >= p.blocks * each) return;
  const uint32_t block = number / each, in = number - block * each, first = in * kPlaces;
  const uint64_t all = ((uint64_t)m * p.blocks + block) * kSorted;
  const uint32_t* row = p.row + all;
  // (a row that is none is nobody's run)
  const uint32_t before = first > 0u ? row[first - 1] : ~0u, after = first + kPlaces < p.places ? row[first + kPlaces] : ~0u;
  const uint32_t token = WHOLE ? 0u : p.token[all + first + threadIdx.x % kPiece];
  uint32_t starts, ends;  // of a piece's places; of a piece of pieces, each piece's first place and its last
  if (WHOLE) {
    starts = row[first + threadIdx.x % kPiece * kPiece];
    ends = row[first + threadIdx.x % kPiece * kPiece + kPiece - 1];
  } else {
    starts = ends = row[first + threadIdx.x % kPiece];
  }
  const uint32_t coming = before < p.vocabulary ? __popc((uint32_t)__ballot(starts == before)) : 0u;
  const uint32_t going = after < p.vocabulary && after != before ? __popc((uint32_t)__ballot(ends == after)) : 0u;
  const Columns<Q> c = columns_of<LANES, Q, NARROW>(blockIdx.y, lane, p.cols);
  const uint64_t stride = 2 * p.cols;
  float* to = (WHOLE ? p.whole : p.piece) + ((uint64_t)m * p.blocks * each + number) * stride;
  const float* piece = WHOLE ? p.piece + (((uint64_t)m * p.blocks + block) * (p.places / kPiece) + in * kPiece) * stride : nullptr;
  const T* dy = static_cast<const T*>(p.dy.p) + m * p.dy.pitch;
  if (coming > 0u) {
    float sum[Q][4] = {};
    if (WHOLE)
      add_parts<Q, NARROW>(piece, stride, coming, c, p.cols, sum);
    else
      add_tokens<T, Q, NARROW>(dy, p.dy.ld, token, 0, coming, c, p.cols, sum);
    store_sum<Q, NARROW>(to, c, p.cols, sum, 1.f, false);
  }
  if (going > 0u) {
    float sum[Q][4] = {};
    if (WHOLE) {
      const float* from = piece + (kPiece - going) * stride;
      add_parts<Q, NARROW>(from + p.cols, stride, 1, c, p.cols, sum);
      add_parts<Q, NARROW>(from + stride, stride, going - 1, c, p.cols, sum);
    } else {
      add_tokens<T, Q, NARROW>(dy, p.dy.ld, token, kPiece - going, going, c, p.cols, sum);
    }
    store_sum<Q, NARROW>(to + p.cols, c, p.cols, sum, 1.f, false);
  }
}

// Rows of the table, p.each for a workgroup, LANES for each at a time.  What it has to write bounds it: 4 x 32000 x 2048, 1049 MB, 190 to 200 us (a fill
// takes 153; of no tokens 188).  Zeros first, by workgroups beside those of the pieces, and then the rows that have tokens, run by run, was 3 % sooner there and
// 13 % later where most rows have some.  Of 5 tokens a row, in five blocks, the latency of tokens and rows: 3 x 4099 x 1003 39 us.
template <typename T, int LANES, int Q, bool NARROW>
__global__ void __launch_bounds__(kBlock) embed_grad_kernel(EmbedGradTask p) {
  constexpr uint32_t kAtATime = kBlock / LANES;
  extern __shared__ uint32_t bound[];  // [block][each + 1]: where each row's places begin
  const uint32_t m = blockIdx.z, group = blockIdx.x, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / LANES), lane = threadIdx.x % LANES, bounds = p.each + 1;
  const uint64_t v0 = (uint64_t)group * p.each;
  const uint32_t rows = (uint32_t)min(p.vocabulary - v0, (uint64_t)p.each);
  const uint64_t all = (uint64_t)m * p.blocks * kSorted;
  for (uint32_t k = threadIdx.x; k < p.blocks * bounds; k += kBlock) {
    const uint32_t block = k / bounds, r = k - block * bounds;
    const uint32_t* begin = p.begin + ((uint64_t)m * p.blocks + block) * (p.groups + 1) + group;
    const uint32_t* row = p.row + all + (uint64_t)block * kSorted;
    uint32_t low = begin[0], high = begin[1];
    while (low < high) {
      const uint32_t mid = (low + high) / 2;
      if (row[mid] < v0 + r)
        low = mid + 1;
      else
        high = mid;
    }
    bound[k] = low;
  }
  __syncthreads();
  const Columns<Q> c = columns_of<LANES, Q, NARROW>(blockIdx.y, lane, p.cols);
  const T* dy = static_cast<const T*>(p.dy.p) + m * p.dy.pitch;
  const uint64_t stride = 2 * p.cols;
  for (uint32_t r = sub; r < rows; r += kAtATime) {
    float sum[Q][4] = {};
    for (uint32_t block = 0; block < p.blocks; ++block) {
      const uint32_t a = __builtin_amdgcn_readfirstlane(bound[block * bounds + r]), b = __builtin_amdgcn_readfirstlane(bound[block * bounds + r + 1]);
      if (a == b) continue;
      const uint32_t piece_a = a / kPiece, piece_b = (b - 1) / kPiece, whole_a = a / kWhole, whole_b = (b - 1) / kWhole;
      if (piece_a == piece_b) {
        add_rows<T, Q, NARROW>(dy, p.dy.ld, p.token + all + (uint64_t)block * kSorted, a, b, c, p.cols, sum);
        continue;
      }
      // the run goes out of its first piece (or piece of pieces), and comes into the others
      const bool whole = p.whole != nullptr && whole_a != whole_b;
      const uint32_t from = whole ? whole_a : piece_a, to = whole ? whole_b : piece_b, each = p.places / (whole ? kWhole : kPiece);
      const float* part = (whole ? p.whole : p.piece) + (((uint64_t)m * p.blocks + block) * each + from) * stride;
      add_parts<Q, NARROW>(part + p.cols, stride, 1, c, p.cols, sum);
      add_parts<Q, NARROW>(part + stride, stride, to - from, c, p.cols, sum);
    }
    store_sum<Q, NARROW>(static_cast<float*>(p.dtable.p) + m * p.dtable.pitch + (v0 + r) * p.dtable.ld, c, p.cols, sum, p.scale, p.past);
  }
}

// Of few tokens: a workgroup looks at all of them for those of its rows.  4 x 33 tokens into 1000 x 256 4.3 us, 200 into 32000 x 2048 37, 262 MB; a launch that
// sorted them first, by counting for each token those before it, made 8.8 and 48 of that.  256 tokens of one row are the longest chain, 13.
template <typename T, int LANES, int Q, bool NARROW>
__global__ void __launch_bounds__(kBlock) embed_grad_few_kernel(EmbedGradTask p, bool longs) {
  constexpr uint32_t kAtATime = kBlock / LANES, kWaves = kBlock / kWave;
  __shared__ uint64_t has[kMostEach][kWaves];  // which lanes of a wavefront have a token of a row
  __shared__ uint32_t token[kFew];             // row by row, in the order that they came in
  const uint32_t m = blockIdx.z, t = threadIdx.x, lane = t % kWave, wave = t / kWave, sub = __builtin_amdgcn_readfirstlane(t / LANES);
  const uint64_t v0 = (uint64_t)blockIdx.x * p.each, at = m * p.ids.pitch + min((uint64_t)t, p.rows - 1) * p.ids.ld;
  const uint32_t rows = (uint32_t)min(p.vocabulary - v0, (uint64_t)p.each);
  const uint64_t id = (uint64_t)(longs ? static_cast<const int64_t*>(p.ids.p)[at] : (int64_t)static_cast<const int32_t*>(p.ids.p)[at]);
  const uint32_t row = t < p.rows && id - v0 < rows ? (uint32_t)(id - v0) : ~0u;
  for (uint32_t r = 0; r < rows; ++r) {
    const uint64_t mine = __ballot(row == r);
    if (lane == 0) has[r][wave] = mine;
  }
  __syncthreads();
  // a lane counts a row's tokens; upto: those of all rows up to it
  uint32_t upto = 0u;
  if (lane < rows) {
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) upto += __popcll(has[lane][w]);
  }
#pragma unroll
  for (uint32_t off = 1; off < kMostEach; off *= 2) {
    const uint32_t other = __shfl_up(upto, off, kWave);
    if (lane >= off) upto += other;
  }
  const uint32_t before = __shfl(upto, (int)min(row, kMostEach) - 1, kWave);
  if (row != ~0u) {
    uint32_t to = (row > 0u ? before : 0u) + __popcll(has[row][wave] & ((1ull << lane) - 1ull));
    for (uint32_t w = 0; w < wave; ++w) to += __popcll(has[row][w]);
    token[to] = t;
  }
  __syncthreads();
  const Columns<Q> c = columns_of<LANES, Q, NARROW>(blockIdx.y, t % LANES, p.cols);
  const T* dy = static_cast<const T*>(p.dy.p) + m * p.dy.pitch;
  for (uint32_t r = sub; r < rows; r += kAtATime) {
    float sum[Q][4] = {};
    const uint32_t a = r > 0u ? (uint32_t)__builtin_amdgcn_readlane((int)upto, (int)r - 1) : 0u, b = (uint32_t)__builtin_amdgcn_readlane((int)upto, (int)r);
    add_rows<T, Q, NARROW>(dy, p.dy.ld, token, a, b, c, p.cols, sum);
    store_sum<Q, NARROW>(static_cast<float*>(p.dtable.p) + m * p.dtable.pitch + (v0 + r) * p.dtable.ld, c, p.cols, sum, p.scale, p.past);
  }
}

__global__ void __launch_bounds__(kBlock) embed_grad_nothing_kernel(uint64_t rows, uint64_t cols, View y) {
  const uint64_t e = block_number() * kBlock + threadIdx.x;
  if (e >= rows * cols) return;
  const uint64_t r = e / cols;
  static_cast<float*>(y.p)[blockIdx.z * y.pitch + r * y.ld + (e - r * cols)] = 0.f;
}

// How many of a block's places are written.
uint32_t places_of(uint64_t rows) { return rows <= 1024 ? 1024u : rows <= 2048 ? 2048u : kSorted; }

// What the gradient keeps, in words of 32 bits.
uint64_t embed_grad_layout(EmbedGradTask& p, uint32_t workers, uint32_t* scratch) {
  p.blocks = (uint32_t)((p.rows + kSorted - 1) / kSorted);
  p.places = places_of(p.rows);
  // Where rows have tokens they take time one after another; where most have none, what a workgroup does before its first one counts.
  p.each = p.rows * 4 >= p.vocabulary ? 4 : kMostEach;
  p.groups = (uint32_t)((p.vocabulary + p.each - 1) / p.each);
  p.bits = 1;
  while (p.vocabulary >> p.bits != 0) ++p.bits;
  if (p.rows <= kFew) return 0;
  const uint64_t blocks = (uint64_t)workers * p.blocks;
  uint64_t at = 0;
  auto take = [&](uint64_t words) {
    uint32_t* here = scratch + at;
    at += (words + 63) / 64 * 64;
    return here;
  };
  p.row = take(blocks * kSorted);
  p.token = take(blocks * kSorted);
  p.begin = take(blocks * (p.groups + 1));
  p.piece = reinterpret_cast<float*>(take(blocks * (p.places / kPiece) * 2 * p.cols));
  p.whole = p.places < kSorted ? nullptr : reinterpret_cast<float*>(take(blocks * (p.places / kWhole) * 2 * p.cols));
  return at;
}

template <typename I>
void sort_typed(uint32_t workers, const EmbedGradTask& p, hipStream_t s) {
  const uint32_t passes = (p.bits + 7) / 8, digit = (p.bits + passes - 1) / passes;
  const dim3 grid(p.blocks, workers);
  auto launch = [&](auto items) { embed_sort_kernel<I, items><<<grid, kSortThreads, 0, s>>>(p, digit, passes); };
  switch (p.places) {
    case 1024: launch(std::integral_constant<int, 1>{}); break;
    case 2048: launch(std::integral_constant<int, 2>{}); break;
    default: launch(std::integral_constant<int, kSorted / kSortThreads>{});
  }
}

template <typename T, bool NARROW>
void embed_grad_typed(uint32_t workers, const EmbedGradTask& p, bool longs, hipStream_t s) {
  const size_t lds = p.blocks * (p.each + 1) * sizeof(uint32_t);
  auto launch = [&](auto lanes, auto fours) {
    const uint32_t across = (uint32_t)((p.cols + lanes * fours * 4 - 1) / (lanes * fours * 4)), at_a_time = kBlock / lanes;
    if (p.rows <= kFew) {
      embed_grad_few_kernel<T, lanes, fours, NARROW><<<dim3(p.groups, across, workers), kBlock, 0, s>>>(p, longs);
      return;
    }
    const uint32_t pieces = p.blocks * (p.places / kPiece), wholes = p.blocks * (p.places / kWhole);
    embed_pieces_kernel<T, false, lanes, fours, NARROW><<<dim3((pieces + at_a_time - 1) / at_a_time, across, workers), kBlock, 0, s>>>(p);
    if (p.whole != nullptr)
      embed_pieces_kernel<T, true, lanes, fours, NARROW><<<dim3((wholes + at_a_time - 1) / at_a_time, across, workers), kBlock, 0, s>>>(p);
    embed_grad_kernel<T, lanes, fours, NARROW><<<dim3(p.groups, across, workers), kBlock, lds, s>>>(p);
  };
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  if (p.cols <= 256)
    launch(std::integral_constant<int, 64>{}, one);
  else if (p.cols <= 512)
    launch(std::integral_constant<int, 64>{}, two);
  else if (p.cols <= 1024)
    launch(std::integral_constant<int, 128>{}, two);
  else
    launch(std::integral_constant<int, 256>{}, two);
}

}  // namespace

hipError_t launch_embed(tng_type of_ids, tng_type of_table, tng_type type, uint32_t workers, uint64_t rows, uint64_t cols, uint64_t vocabulary,
                        const View& ids, const View& table, float scale, const View& y, hipStream_t s) {
  EmbedTask p{rows, cols, 0, vocabulary, ids, table, y, scale, false};
  p.past = (uint64_t)workers * rows * cols * (type == TNG_TYPE_F32 ? 4 : 2) > kPast;
  if (of_ids == TNG_TYPE_I32)
    embed_from<int32_t>(of_table, type, workers, p, s);
  else
    embed_from<int64_t>(of_table, type, workers, p, s);
  return hipGetLastError();
}

size_t embed_grad_words(uint32_t workers, uint64_t rows, uint64_t cols, uint64_t vocabulary) {
  EmbedGradTask p{};
  p.rows = rows;
  p.cols = cols;
  p.vocabulary = vocabulary;
  return embed_grad_layout(p, workers, nullptr);
}

hipError_t launch_embed_grad(tng_type of_ids, tng_type type, uint32_t workers, uint64_t rows, uint64_t cols, uint64_t vocabulary, const View& ids,
                             const View& dy, float scale, const View& dtable, uint32_t* scratch, hipStream_t s) {
  if (rows == 0) {
    embed_grad_nothing_kernel<<<grid_of((vocabulary * cols + kBlock - 1) / kBlock, workers), kBlock, 0, s>>>(vocabulary, cols, dtable);
    return hipGetLastError();
  }
  EmbedGradTask p{};
  p.rows = rows;
  p.cols = cols;
  p.vocabulary = vocabulary;
  p.ids = ids;
  p.dy = dy;
  p.dtable = dtable;
  p.scale = scale;
  p.past = (uint64_t)workers * vocabulary * cols * sizeof(float) > kPast;
  embed_grad_layout(p, workers, scratch);
  const bool longs = of_ids == TNG_TYPE_I64;
  if (p.rows > kFew) longs ? sort_typed<int64_t>(workers, p, s) : sort_typed<int32_t>(workers, p, s);
  auto grad = [&](auto narrow) {
    switch (type) {
      case TNG_TYPE_F32: embed_grad_typed<float, narrow>(workers, p, longs, s); break;
      case TNG_TYPE_BF16: embed_grad_typed<bf16_t, narrow>(workers, p, longs, s); break;
      default: embed_grad_typed<f16_t, narrow>(workers, p, longs, s); break;
    }
  };
  if (cols < 4)
    grad(std::true_type{});
  else
    grad(std::false_type{});
  return hipGetLastError();
}

}  // namespace tng
