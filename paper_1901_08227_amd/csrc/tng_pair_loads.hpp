// What a workgroup's loads of one operand's rows touch.  Plain arithmetic, the same on the host.
#pragma once

#include <cstdint>

namespace tng {

// Rows of one operand that a tile has, and the stages (128 bytes of every row) that it has not asked for.  A load takes 16 bytes for each lane, eight lanes a
// row: eight rows for a wavefront, from a row that is the same for all of them.  It is held in bounds by its descriptor alone: base and bytes say where its
// rows begin and what there is from there to the end of the last one, and a lane whose offset is no less than that reads nothing.  (Rows that all loads but the
// first begin at are no scalar offset: what the units make of one beyond `bytes` is not said anywhere.)
struct PairRows {
  uint64_t base;   // the first row, at the first stage that has not been asked for
  uint32_t bytes;  // from there to the end of the last row's stages; none left: 0
  uint32_t ld;     // from row to row
  int32_t left;    // stages that have not been asked for

  // all: the operand's rows; first, count: of a tile of them; stage, stages: those of its depth.
  __host__ __device__ static PairRows of(uint64_t p, uint64_t ld, uint32_t all, uint32_t first, uint32_t count, uint32_t stage, uint32_t stages) {
    const uint32_t rows = all - first < count ? all - first : count;
    return PairRows{p + first * ld + stage * 128ull, (rows - 1) * (uint32_t)ld + stages * 128u, (uint32_t)ld, (int32_t)stages};
  }
  __host__ __device__ uint32_t offset(uint32_t lane, uint32_t wave) const {
    const uint32_t r = wave * 8 + lane / 8;
    return r * ld + (lane % 8 ^ (r >> 1 & 7u)) * 16;  // (rows that loads are apart do not change what pieces are moved by)
  }
  struct Descriptor {
    uint64_t base;
    uint32_t bytes;
  };
  // Of the load whose first wavefront's rows begin at `row`.
  __host__ __device__ Descriptor from(uint32_t row) const {
    const uint32_t skip = row * ld;
    const int32_t rest = (int32_t)(bytes - skip);  // (below 2^31: 256 rows of 256 KB)
    return Descriptor{base + skip, (uint32_t)(rest > 0 ? rest : 0)};
  }
  __host__ __device__ void next() {
    --left;
    base += 128;
    bytes = left > 0 ? bytes - 128 : 0;
  }
};

}  // namespace tng
