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

struct EmbedTask {
  uint64_t rows, cols, eights;  // tokens of a worker; columns; lanes that a row takes
  uint64_t vocabulary;
  View ids, table, y;
  float scale;
};

// y = scale table[id].  A lane takes eight columns of kMany tokens' rows (the row's last eight where it ends inside them: what two lanes write of
// one column is the same), so that their tokens, and then their rows, are on the way together.
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
    t[k] = n >> 32 == 0 ? (uint32_t)at / (uint32_t)p.eights : at / p.eights;  // (64 bits take four times the instructions)
    c[k] = (at - t[k] * p.eights) * 8;
    if (!NARROW) c[k] = min(c[k], p.cols - 8);
    row[k] = row_of<I>(ids, t[k] * p.ids.ld, p.vocabulary);
  }
  Vec8<W> w[kMany];
#pragma unroll
  for (int k = 0; k < kMany; ++k) {
    const W* from = table + (uint64_t)(row[k] < p.vocabulary ? row[k] : 0u) * p.table.ld + c[k];
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
    } else {
      *reinterpret_cast<Vec8<T>*>(to) = v;
    }
  }
}

// No row to read: all tokens are outside.
template <typename T>
__global__ void __launch_bounds__(kBlock) embed_nothing_kernel(uint64_t rows, uint64_t cols, View y) {
  const uint64_t e = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
  if (e >= rows * cols) return;
  const uint64_t r = e / cols;
  static_cast<T*>(y.p)[blockIdx.y * y.pitch + r * y.ld + (e - r * cols)] = (T)0.f;
}

template <typename I, typename W, typename T>
void embed_typed(uint32_t workers, EmbedTask& p, hipStream_t s) {
  if (p.vocabulary == 0) {
    embed_nothing_kernel<T><<<dim3((uint32_t)((p.rows * p.cols + kBlock - 1) / kBlock), workers), kBlock, 0, s>>>(p.rows, p.cols, p.y);
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
// together then, in the order that they came in, whatever ran first.  Sums are taken in that order: of pieces of kPiece sorted places that are
// all one row's (for rows that many tokens ask for), of kPiece such pieces, and then of a row.  Every row of the table is written, those of no token with zeros.
constexpr uint32_t kSorted = 8192, kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr uint32_t kPiece = 32, kWhole = kPiece * kPiece;  // places of a piece, and of a piece of pieces
constexpr uint32_t kRowsOfGroup = 16;                       // rows of the table that a workgroup writes
constexpr uint32_t kMostBins = 256;

struct EmbedGradTask {
  uint64_t rows, cols, vocabulary;
  View ids, dy, dtable;
  float scale;
  uint32_t bits;          // of a row's number; the largest number they hold stands for no row
  uint32_t blocks;        // of kSorted tokens, of a worker
  uint32_t groups;        // of rows of the table
  uint32_t *row, *token;  // [worker][blocks kSorted]: sorted rows, and the token's number
  uint32_t* begin;        // [worker][block][groups + 1]: where a group's rows begin in a block
  float *piece, *whole;   // [worker][blocks kSorted / kPiece][cols], and / kWhole
};

// Least significant digits first, of 2^digit bins.  A wavefront takes consecutive places, 64 at a time: lanes of one digit find each other by ballots, and
// the wavefront's counter of that digit says how many came before them.  That all is in one CU's LDS is what bounds it.
template <typename I, int ITEMS>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(EmbedGradTask p, uint32_t digit, uint32_t passes) {
  __shared__ uint32_t keys[ITEMS * kSortThreads];
  __shared__ uint16_t from[ITEMS * kSortThreads];
  __shared__ uint32_t count[kMostBins][kSortWaves + 1];  // (one more: the bins of a wavefront lie in different banks)
  __shared__ uint32_t of_wave[kSortWaves];
  const uint32_t m = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, bins = 1u << digit;
  const uint64_t first = (uint64_t)blockIdx.x * kSorted;
  const I* ids = static_cast<const I*>(p.ids.p) + m * p.ids.pitch;
  const uint32_t none = p.bits < 32 ? (1u << p.bits) - 1u : ~0u, base = wave * (ITEMS * kWave) + lane;
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
  // where each group of rows begins: the first place whose row is no less
  for (uint32_t g = threadIdx.x; g <= p.groups; g += kSortThreads) {
    const uint64_t want = min((uint64_t)g * kRowsOfGroup, p.vocabulary);
    uint32_t low = 0u, high = ITEMS * kSortThreads;
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

// Eight columns of the rows of `token`s first .. end - 1 added to sum, kMany rows on the way at a time.
template <typename T, bool NARROW>
__device__ __forceinline__ void add_rows(const T* dy, uint64_t ld, const uint32_t* token, uint32_t first, uint32_t end, uint64_t cols, float (&sum)[8]) {
  constexpr uint32_t kMany = 8;
  for (; first < end; first += kMany) {
    Vec8<T> v[kMany];
#pragma unroll
    for (uint32_t k = 0; k < kMany; ++k) {  // (past the end: the last one again, which is not counted)
      const T* row = dy + (uint64_t)token[min(first + k, end - 1)] * ld;
      if (NARROW) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[k][i] = i < cols ? row[i] : (T)0.f;
      } else {
        v[k] = *reinterpret_cast<GlobalPtr<Vec8<T>>>((GlobalPtr<T>)row);
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < kMany; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += first + k < end ? (float)v[k][i] : 0.f;
  }
}

template <bool NARROW>
__device__ __forceinline__ void add_parts(const float* part, uint64_t cols, uint32_t count, float (&sum)[8]) {
  constexpr uint32_t kMany = 8;
  for (uint32_t first = 0; first < count; first += kMany) {
    Vec8<float> v[kMany];
#pragma unroll
    for (uint32_t k = 0; k < kMany; ++k) {
      const float* row = part + (uint64_t)min(first + k, count - 1) * cols;
      if (NARROW) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[k][i] = i < cols ? row[i] : 0.f;
      } else {
        v[k] = *reinterpret_cast<GlobalPtr<Vec8<float>>>((GlobalPtr<float>)row);
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < kMany; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += first + k < count ? v[k][i] : 0.f;
  }
}

template <bool NARROW>
__device__ __forceinline__ void store_sum(float* to, uint64_t cols, const float (&sum)[8], float scale) {
  Vec8<float> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = sum[i] * scale;
  if (NARROW) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < cols) to[i] = v[i];
  } else {
    *reinterpret_cast<Vec8<float>*>(to) = v;
  }
}

// Pieces (or pieces of pieces) that are all one row's: their sums.  The others are not looked at.
template <typename T, bool WHOLE, bool NARROW>
__global__ void __launch_bounds__(kBlock) embed_pieces_kernel(EmbedGradTask p) {
  constexpr uint32_t kPlaces = WHOLE ? kWhole : kPiece;
  const uint32_t m = blockIdx.z, number = blockIdx.x;
  const uint64_t at = (uint64_t)m * p.blocks * kSorted, first = (uint64_t)number * kPlaces;
  const uint32_t row = p.row[at + first];
  if (row >= p.vocabulary || p.row[at + first + kPlaces - 1] != row) return;
  uint64_t c = ((uint64_t)blockIdx.y * kBlock + threadIdx.x) * 8;
  if (c >= p.cols) return;
  if (!NARROW) c = min(c, p.cols - 8);
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const uint64_t pieces = (uint64_t)p.blocks * (kSorted / kPiece), wholes = (uint64_t)p.blocks * (kSorted / kWhole);
  if (WHOLE) {
    add_parts<NARROW>(p.piece + (m * pieces + number * kPiece) * p.cols + c, p.cols, kPiece, sum);
    store_sum<NARROW>(p.whole + (m * wholes + number) * p.cols + c, p.cols, sum, 1.f);
  } else {
    add_rows<T, NARROW>(static_cast<const T*>(p.dy.p) + m * p.dy.pitch + c, p.dy.ld, p.token + at + first, 0, kPiece, p.cols, sum);
    store_sum<NARROW>(p.piece + (m * pieces + number) * p.cols + c, p.cols, sum, 1.f);
  }
}

// Rows of the table, kRowsOfGroup for a workgroup, LANES for each at a time.  What it has to write bounds it.
template <typename T, int LANES, bool NARROW>
__global__ void __launch_bounds__(kBlock) embed_grad_kernel(EmbedGradTask p) {
  constexpr uint32_t kAtATime = kBlock / LANES;
  extern __shared__ uint32_t bound[];  // [block][kRowsOfGroup + 1]: where each row's places begin
  const uint32_t m = blockIdx.z, group = blockIdx.x, sub = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const uint64_t v0 = (uint64_t)group * kRowsOfGroup;
  const uint32_t rows = (uint32_t)min(p.vocabulary - v0, (uint64_t)kRowsOfGroup);
  const uint64_t all = (uint64_t)m * p.blocks * kSorted;
  for (uint32_t k = threadIdx.x; k < p.blocks * (kRowsOfGroup + 1); k += kBlock) {
    const uint32_t block = k / (kRowsOfGroup + 1), r = k - block * (kRowsOfGroup + 1);
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
  uint64_t c = ((uint64_t)blockIdx.y * LANES + lane) * 8;
  if (c >= p.cols) return;
  if (!NARROW) c = min(c, p.cols - 8);
  const T* dy = static_cast<const T*>(p.dy.p) + m * p.dy.pitch + c;
  const uint64_t pieces = (uint64_t)p.blocks * (kSorted / kPiece), wholes = (uint64_t)p.blocks * (kSorted / kWhole);
  for (uint32_t r = sub; r < rows; r += kAtATime) {
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (uint32_t block = 0; block < p.blocks; ++block) {
      uint32_t a = bound[block * (kRowsOfGroup + 1) + r];
      const uint32_t b = bound[block * (kRowsOfGroup + 1) + r + 1];
      const uint32_t* token = p.token + all + (uint64_t)block * kSorted;
      // tokens up to a whole piece, pieces up to a piece of pieces, those, and the same down again
      const uint32_t piece_a = (a + kPiece - 1) / kPiece, piece_b = b / kPiece;
      if (piece_a >= piece_b) {
        add_rows<T, NARROW>(dy, p.dy.ld, token, a, b, p.cols, sum);
        continue;
      }
      add_rows<T, NARROW>(dy, p.dy.ld, token, a, piece_a * kPiece, p.cols, sum);
      const float* piece = p.piece + (m * pieces + block * (kSorted / kPiece)) * p.cols + c;
      const uint32_t whole_a = (piece_a + kPiece - 1) / kPiece, whole_b = piece_b / kPiece;
      if (whole_a >= whole_b) {
        add_parts<NARROW>(piece + (uint64_t)piece_a * p.cols, p.cols, piece_b - piece_a, sum);
      } else {
        add_parts<NARROW>(piece + (uint64_t)piece_a * p.cols, p.cols, whole_a * kPiece - piece_a, sum);
        add_parts<NARROW>(p.whole + (m * wholes + block * (kSorted / kWhole) + whole_a) * p.cols + c, p.cols, whole_b - whole_a, sum);
        add_parts<NARROW>(piece + (uint64_t)whole_b * kPiece * p.cols, p.cols, piece_b - whole_b * kPiece, sum);
      }
      add_rows<T, NARROW>(dy, p.dy.ld, token, piece_b * kPiece, b, p.cols, sum);
    }
    store_sum<NARROW>(static_cast<float*>(p.dtable.p) + m * p.dtable.pitch + (v0 + r) * p.dtable.ld + c, p.cols, sum, p.scale);
  }
}

__global__ void __launch_bounds__(kBlock) embed_grad_nothing_kernel(uint64_t rows, uint64_t cols, View y) {
  const uint64_t e = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
  if (e >= rows * cols) return;
  const uint64_t r = e / cols;
  static_cast<float*>(y.p)[blockIdx.y * y.pitch + r * y.ld + (e - r * cols)] = 0.f;
}

// What the gradient keeps, in words of 32 bits.
uint64_t embed_grad_layout(EmbedGradTask& p, uint32_t workers, uint32_t* scratch) {
  p.blocks = (uint32_t)((p.rows + kSorted - 1) / kSorted);
  p.groups = (uint32_t)((p.vocabulary + kRowsOfGroup - 1) / kRowsOfGroup);
  p.bits = 1;
  while (p.bits < 32 && p.vocabulary >> p.bits != 0) ++p.bits;
  const uint64_t places = (uint64_t)workers * p.blocks * kSorted;
  uint64_t at = 0;
  auto take = [&](uint64_t words) {
    uint32_t* here = scratch + at;
    at += (words + 63) / 64 * 64;
    return here;
  };
  p.row = take(places);
  p.token = take(places);
  p.begin = take((uint64_t)workers * p.blocks * (p.groups + 1));
  const bool pieces = p.rows >= kPiece, wholes = p.rows >= kWhole;
  p.piece = reinterpret_cast<float*>(take(pieces ? places / kPiece * p.cols : 0));
  p.whole = reinterpret_cast<float*>(take(wholes ? places / kWhole * p.cols : 0));
  return at;
}

template <typename I>
void sort_typed(uint32_t workers, const EmbedGradTask& p, hipStream_t s) {
  const uint32_t passes = (p.bits + 7) / 8, digit = (p.bits + passes - 1) / passes;
  const dim3 grid(p.blocks, workers);
  auto launch = [&](auto items) { embed_sort_kernel<I, items><<<grid, kSortThreads, 0, s>>>(p, digit, passes); };
  if (p.rows <= 1024)
    launch(std::integral_constant<int, 1>{});
  else if (p.rows <= 2048)
    launch(std::integral_constant<int, 2>{});
  else if (p.rows <= 4096)
    launch(std::integral_constant<int, 4>{});
  else
    launch(std::integral_constant<int, 8>{});
}

template <typename T, bool NARROW>
void embed_grad_typed(uint32_t workers, const EmbedGradTask& p, hipStream_t s) {
  const uint64_t eights = (p.cols + 7) / 8;
  const uint32_t across = (uint32_t)((eights + kBlock - 1) / kBlock);
  // (places behind the last sorted ones of a short block are never written, and belong to no piece that is looked at)
  const uint32_t places = (uint32_t)(p.rows <= 4096 ? (p.rows + kSortThreads - 1) / kSortThreads * kSortThreads : (uint64_t)p.blocks * kSorted);
  if (p.rows >= kPiece) embed_pieces_kernel<T, false, NARROW><<<dim3(std::min<uint32_t>(places / kPiece, (uint32_t)(p.rows / kPiece) + 1), across, workers), kBlock, 0, s>>>(p);
  if (p.rows >= kWhole) embed_pieces_kernel<T, true, NARROW><<<dim3(places / kWhole, across, workers), kBlock, 0, s>>>(p);
  const size_t lds = p.blocks * (kRowsOfGroup + 1) * sizeof(uint32_t);
  auto launch = [&](auto lanes) {
    embed_grad_kernel<T, lanes, NARROW><<<dim3(p.groups, (uint32_t)((eights + lanes - 1) / lanes), workers), kBlock, lds, s>>>(p);
  };
  if (eights <= 64)
    launch(std::integral_constant<int, 64>{});
  else if (eights <= 128)
    launch(std::integral_constant<int, 128>{});
  else
    launch(std::integral_constant<int, 256>{});
}

}  // namespace

hipError_t launch_embed(tng_type of_ids, tng_type of_table, tng_type type, uint32_t workers, uint64_t rows, uint64_t cols, uint64_t vocabulary,
                        const View& ids, const View& table, float scale, const View& y, hipStream_t s) {
  EmbedTask p{rows, cols, 0, vocabulary, ids, table, y, scale};
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
    embed_grad_nothing_kernel<<<dim3((uint32_t)((vocabulary * cols + kBlock - 1) / kBlock), workers), kBlock, 0, s>>>(vocabulary, cols, dtable);
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
  embed_grad_layout(p, workers, scratch);
  if (of_ids == TNG_TYPE_I32)
    sort_typed<int32_t>(workers, p, s);
  else
    sort_typed<int64_t>(workers, p, s);
  auto grad = [&](auto narrow) {
    switch (type) {
      case TNG_TYPE_F32: embed_grad_typed<float, narrow>(workers, p, s); break;
      case TNG_TYPE_BF16: embed_grad_typed<bf16_t, narrow>(workers, p, s); break;
      default: embed_grad_typed<f16_t, narrow>(workers, p, s); break;
    }
  };
  if (cols < 8)
    grad(std::true_type{});
  else
    grad(std::false_type{});
  return hipGetLastError();
}

}  // namespace tng
