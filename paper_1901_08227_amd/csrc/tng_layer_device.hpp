// Device helpers shared by the layer kernels: element types, dropout's and the rounding's draws, 8-bit codes.
#pragma once

#include "tng_device.hpp"
#include "tng_layer_kernels.hpp"

namespace tng {

using bf16_t = __bf16;
using f16_t = _Float16;

// A number of 32 bits as it is.  (An operation and the conversion of its result to 16 bits may become one instruction, which rounds once: where results are
// compared bit for bit they are two.)
__device__ __forceinline__ float pinned(float x) {
  asm("" : "+v"(x));
  return x;
}

// Workgroups by one number, of up to 1024 threads each: a grid's side holds 2^32 threads less one, which rows of the longest matrices pass.
inline dim3 grid_of(uint64_t blocks, uint32_t workers = 1) {
  const uint64_t side = 1u << 20;
  return dim3((uint32_t)(blocks < side ? blocks : side), (uint32_t)((blocks + side - 1) / side), workers);
}
__device__ __forceinline__ uint64_t block_number() { return (uint64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Eight (or N) consecutive elements at an address of the element's own alignment, as 32-bit numbers.  Rows of odd length start
// anywhere; loads of 16 bytes are legal there on this target.
template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, float (&out)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(alignof(T))));
  const vec v = *reinterpret_cast<GlobalPtr<vec>>((GlobalPtr<T>)p);
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = (float)v[i];
}

// The same where only the first `count` exist; the others are `fill`.
template <typename T, int N>
__device__ __forceinline__ void load_n_within(const T* p, uint64_t count, float fill, float (&out)[N]) {
  if (count >= N) {
    load_n<T, N>(p, out);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = (uint64_t)i < count ? (float)p[i] : fill;
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_n_within(T* p, uint64_t count, const float (&x)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(alignof(T))));
  if (count >= N) {
    vec v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    *reinterpret_cast<vec*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((uint64_t)i < count) p[i] = (T)x[i];
  }
}

// The words of elements e .. e + N - 1 (N a multiple of 4) of a worker.  Where e is no multiple of 4 they begin inside a block:
// one block more is drawn and the words are moved down.  aligned: e is a multiple of 4 in every lane.
template <int N>
__device__ __forceinline__ void draw_n(uint64_t e, bool aligned, uint32_t worker, const DropArgs& d, uint32_t (&word)[N]) {
  const uint32_t block = (uint32_t)(e >> 2);
#pragma unroll
  for (int b = 0; b < N / 4; ++b) {
    const U32x4 w = philox4x32_10(block + b, worker, d.iter, d.word, d.k0, d.k1);
    word[4 * b] = w.x;
    word[4 * b + 1] = w.y;
    word[4 * b + 2] = w.z;
    word[4 * b + 3] = w.w;
  }
  if (!aligned) {
    const U32x4 w = philox4x32_10(block + N / 4, worker, d.iter, d.word, d.k0, d.k1);
    const uint32_t by = (uint32_t)e & 3u;
    const uint32_t last[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t a0 = word[i], a1 = i + 1 < N ? word[i + 1] : last[i + 1 - N], a2 = i + 2 < N ? word[i + 2] : last[i + 2 - N],
                     a3 = i + 3 < N ? word[i + 3] : last[i + 3 - N];
      word[i] = by < 2u ? (by == 0u ? a0 : a1) : (by == 2u ? a2 : a3);
    }
  }
}

__device__ __forceinline__ bool kept(uint32_t word, const DropArgs& d) { return word >= d.threshold; }

// relu that lets NaN through.
__device__ __forceinline__ float relu(float x) { return x < 0.f ? 0.f : x; }

// What the layer in front of a product hands on: keep f(x) / (1 - p).
__device__ __forceinline__ float dropped(float x, uint32_t word, const DropArgs& d) {
  const float f = (d.relu ? relu(x) : x) * d.scale;
  return kept(word, d) ? f : 0.f;
}

// ---- 8-bit codes.  R: the largest magnitude, as the bits of a number without sign (NaN above infinity, so that neither is lost).
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t x) {
  int v = (int)x;
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x140, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xA, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xC, 0xF, false));
  return (uint32_t)__builtin_amdgcn_readlane(v, 63);
}

// 1 / R, or 0 where R is below the smallest normal number (all codes are 0 then) or no finite number.
__device__ __forceinline__ float code_inverse(uint32_t r) {
  return r < 0x00800000u || r >= 0x7F800000u ? 0.f : 1.0f / __uint_as_float(r);
}
// What a code of 1 stands for; NaN where the row holds what is not finite.
__device__ __forceinline__ float code_step(uint32_t r) {
  if (r < 0x00800000u) return 0.f;
  return r >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(r) / 127.0f;
}

// v on the scale of codes, -127 .. 127: two roundings.
__device__ __forceinline__ float code_place(float v, float inv) {
  return __builtin_amdgcn_fmed3f(v * inv, -1.0f, 1.0f) * 127.0f;
}
// Its code is the lowest byte.  (1.5 2^23 leaves no place for a fraction: the sum is rounded to the nearest integer, halves to even.)
__device__ __forceinline__ uint32_t code_nearest(float v, float inv) { return __float_as_uint(code_place(v, inv) + 0x1.8p23f); }
// Up with the probability of the fractional part, to 2^-16 of a step (of a code: the mean is within 2^-16 of a step of v).  The code is the
// lowest byte.  (v_fract gives x - floor(x), but no more than 1 - 2^-24; no draw lies between that and 1.)
__device__ __forceinline__ uint32_t code_drawn(float v, float inv, uint32_t half) {
  const float x = code_place(v, inv);
  return (uint32_t)((int)floorf(x) + ((float)half * 0x1p-16f < __builtin_amdgcn_fractf(x) ? 1 : 0));
}

// The lowest bytes of four words as one.
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

// x and the lane's that a data-parallel control names, in the rows of 16 lanes that ROWS has.
template <int CTRL, int ROWS>
__device__ __forceinline__ float plus_other(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xF, false));
}

// ---- Tiles of the products: loads that go to LDS directly.
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// 16 (4) bytes for each lane, from base + its offset to LDS, one lane's behind the other from `lds` on; what lies past `bytes` reads as 0.
// The compiler does not count these loads: wait_and_meet does.  (s_mov and s_nop 3: as long as a scalar register written by the vector unit needs.)
__device__ __forceinline__ void load_to_lds(uint64_t base, uint32_t bytes, uint32_t offset, uint32_t lds) {
  const v4u rsrc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, bytes, 0x00020000u};
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds"
      :
      : "s"(lds), "v"(offset), "s"(rsrc)
      : "memory");
}
__device__ __forceinline__ void load_words_to_lds(uint64_t base, uint32_t bytes, uint32_t offset, uint32_t lds) {
  const v4u rsrc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, bytes, 0x00020000u};
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dword %1, %2, 0 offen lds"
      :
      : "s"(lds), "v"(offset), "s"(rsrc)
      : "memory");
}

// All but the last `left` loads of every wavefront are in LDS, and every wavefront has what it reads there.
template <int left>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(left) : "memory");
}

}  // namespace tng
